"""wt.adapt_array: what a kept array of descriptors holds."""
import ctypes as C
import gc
import weakref

from paper_2608_12114_gb300 import wt


def test_an_array_of_descriptors_holds_what_they_hold():
    class Tensor:
        pass

    t = Tensor()
    d = wt.AdaptDesc(T=7)
    d.tensors = (t,)
    alive = weakref.ref(t)
    a = wt.adapt_array([d, d])
    del d, t
    gc.collect()
    assert alive() is not None and len(a) == 2 and a[1].T == 7 and isinstance(a, C.Array)
    del a
    gc.collect()
    assert alive() is None
