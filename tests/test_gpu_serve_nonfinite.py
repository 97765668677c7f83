"""A serving step's operators beside NaN, infinities and weights of very different sizes: what an element
may reach it reaches on every route, and what it may not it does not."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve
from tests.test_gpu_serve_adapt import close, make
from tests.test_gpu_serve_attend import Set

pytestmark = pytest.mark.gpu
NAN, INF = _serve.NAN, _serve.INF


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


def fill_workspace_with_nan(torch, h):
    """A call whose partial results are NaN, 57 KB of them, on the stream the next call uses."""
    s = Set(torch, [1], None, 500, 14, 2, 128)
    s.q.fill_(NAN)
    h.attend(s.desc())


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("R,rank", [(8, [0, 8]), (8, [-2, 5]), (0, None)])
def test_slots_of_rank_zero_among_many_tokens(torch, dt, R, rank):
    """Nothing of the workspace reaches y, whatever it held."""
    x, y, slot, A, B, scale, base = make(torch, 300, 96, 48, 2, R, getattr(torch, dt))
    rk = None if rank is None else torch.tensor(rank, dtype=torch.int32, device="cuda")
    with wt.Handle([]) as h:
        fill_workspace_with_nan(torch, h)
        h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=rk, base=base)])
        torch.cuda.synchronize()
        close(torch, y, _serve.adapt(x, slot, A, B, scale, rk, base), 96, R)
