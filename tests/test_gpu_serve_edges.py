"""Placing and attention to memories at the edges of what a call may hold: parts without the rest, the most rows."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests.test_gpu_serve_cross import Set as Cross
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


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("rise", [0.0, 1.3, 5.2])
@pytest.mark.parametrize("new,D", [([1, 2], 64), ([1, 2], 128), ([16, 9], 128), ([20, 30], 64), ([20, 30], 128), ([200, 3], 64), ([200, 3], 128)])
def test_roundings_that_weights_share_cancel_on_every_route(torch, h, dt, rise, new, D):
    """Scores of two kinds, so that most weights are one number and share its rounding: it must not show in
    the result, which then errs to both sides alike (128 different columns and more, whose roundings have a
    variance of u^2 / 3 at most: a mean error of 0.2 u would be four standard deviations of these alone)."""
    s = Cross(torch, new, [4000] * len(new), 4, 2, D, dt=dt, sharp=0.0)
    s.q[:, :, 0] = 1.0
    s.scale = 1.0
    M = s.k.shape[0]
    steps = rise * (torch.arange(M, device="cuda") // 128 % 2).view(-1, 1).to(s.k.dtype)
    s.k[:, :, 0] = torch.where(s.inside.view(-1, 1), steps, s.k[:, :, 0])
    s.v += torch.linspace(1, 8, 2 * D, device="cuda").view(2, D).to(s.v.dtype)
    h.cross(s.desc())
    torch.cuda.synchronize()
    o, _, _ = s.want()
    off = (s.out.double().cpu() - o) / o
    assert off.abs().max() <= 1.1 * s.u and off.mean().abs() <= 0.2 * s.u
