"""Placing and attention to memories at the edges of what a call may hold: parts without the rest, the most rows."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests.test_gpu_serve_place import Set as Place

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


@pytest.mark.parametrize("src,D", [("f32", 64), ("bf16", 64), ("bf16", 72)])
def test_values_alone_need_no_turns(torch, h, src, D):
    """Values are placed as they are, whatever a rotation that nobody asks for would need."""
    s = Place(torch, [3, 1], [2, 15], parts="v", src=src, D=D, rot=D)
    d = s.desc()
    d.turns, d.pos, d.pos_stride, d.axes = None, None, 0, 0
    d.axis[:] = [255] * len(d.axis)
    h.place(d)
    s.check(torch)


@pytest.mark.parametrize("heads", [2, 128])
@pytest.mark.parametrize("scale", [0.0, 1.0])  # on the warp kernel and on tcgen05
def test_rows_up_to_2_31(torch, h, heads, scale):
    """One request of as many rows as a call may have, to one state: every row becomes that state's value."""
    N, D = (2 ** 31 - 1) // heads, 8
    q = torch.zeros(N, heads, D, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.tensor([x], dtype=torch.bfloat16, device="cuda").view(1, 1, D) for x in ([0] * D, range(1, D + 1)))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    h.cross(serving.cross_attention(q, q, ints(0, N), k, v, ints(0), ints(1), max_new=N, max_mem=1, scale=scale))
    torch.cuda.synchronize()
    rows = q.view(-1, D)
    for i in range(0, len(rows), 1 << 28):
        assert (rows[i:i + (1 << 28)] == v.view(1, D)).all(), i
    del q, rows
    torch.cuda.empty_cache()
