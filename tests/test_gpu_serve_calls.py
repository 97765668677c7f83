"""How a program makes the serving calls: from threads and streams, into graphs, many at a time, again and again."""
import ctypes as C

import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests.test_gpu_serve_adapt import make
from tests.test_gpu_serve_attend import Set

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    build.build()
    wt.lib()
    return torch


@pytest.fixture()
def h(torch):
    with wt.Handle([]) as h:
        yield h
        torch.cuda.synchronize()
        assert h.device_status() == 0


def test_the_first_kernel_of_a_call_waits_for_the_stream(torch, h):
    """In a capture, the edge to a call's first kernel from what came before it is a full one: only the
    kernels within a call follow one another programmatically."""
    rt = C.CDLL("libcudart.so.13")
    rt.cudaStreamBeginCapture.argtypes = [C.c_void_p, C.c_int]
    rt.cudaStreamEndCapture.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
    rt.cudaGraphGetEdges.argtypes = [C.c_void_p] + [C.c_void_p] * 4
    rt.cudaGraphDestroy.argtypes = [C.c_void_p]
    x = make(torch, 300, 64, 32, 2, 8, torch.bfloat16)
    sets = [Set(torch, [2, 1], None, 0, 4, 2, 64), Set(torch, [2, 1], [40, 33], 0, 4, 2, 64), Set(torch, [2, 1], [40, 33], 900, 4, 2, 64),
            Set(torch, [2] * 20, [9] * 20, 900, 4, 2, 64), Set(torch, [2] * 20, None, 900, 4, 2, 64)]
    calls = [lambda st, s=s: h.attend(s.desc(), st) for s in sets]  # the first: no key at all
    calls.append(lambda st: h.adapt([serving.adapters(x[0], x[1], x[2], x[3], x[4], x[5], base=x[6])], st))
    mark = torch.zeros(4, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call in calls:
        g, n = C.c_void_p(), C.c_size_t()
        assert rt.cudaStreamBeginCapture(st.cuda_stream, 2) == 0
        try:
            with torch.cuda.stream(st):
                mark.fill_(1.0)
            call(st.cuda_stream)
        finally:
            assert rt.cudaStreamEndCapture(st.cuda_stream, C.byref(g)) == 0
        assert rt.cudaGraphGetEdges(g, None, None, None, C.byref(n)) == 0 and n.value >= 1
        frm, to, data = (C.c_void_p * n.value)(), (C.c_void_p * n.value)(), (C.c_uint8 * (8 * n.value))()
        assert rt.cudaGraphGetEdges(g, frm, to, data, C.byref(n)) == 0
        first = set(frm) - set(to)
        assert len(first) == 1
        kinds = [data[8 * i + 2] for i in range(n.value) if frm[i] in first]
        assert kinds == [0], kinds
        rt.cudaGraphDestroy(g)
