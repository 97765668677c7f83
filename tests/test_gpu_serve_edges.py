"""Placing at the edges of what a call may hold: parts without the rest."""
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
