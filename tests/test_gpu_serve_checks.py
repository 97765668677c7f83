"""What a serving call refuses and accepts by its descriptors, and what it reports of values in device memory."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve
from tests.test_gpu_serve_adapt import close, make
from tests.test_gpu_serve_attend import Set
from tests.test_gpu_serve_draw import drafts

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


def refused(call, desc, says=""):
    with pytest.raises(wt.WtError) as e:
        call(desc)
    assert e.value.code == wt.WT_EINVAL and says in str(e.value), str(e.value)


def test_sizes_whose_bytes_pass_64_bits(torch, h):
    """Products that come round to a small number must not pass for one."""
    l, p = torch.randn(3, 64, device="cuda"), torch.empty(3, 64, device="cuda")
    d = serving.probabilities(l, p)
    d.rows, d.ldl, d.ldp = (1 << 26) + 1, 1 << 36, 1 << 36
    refused(h.probs, d, "logits runs past")
    a = drafts(torch, [2, 1], 64, 1.0, False)
    acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    d = serving.verification(a[0], a[2], a[3], a[4], a[5], acc, tok, q=a[1])
    d.ldp, d.n_drafted = 1 << 40, (1 << 22) - 1
    refused(h.verify, d, "p runs past")
    x, y, slot, A, B, scale, base = make(torch, 4, 64, 32, 2, 8, torch.bfloat16)
    d = serving.adapters(x, y, slot, A, B, scale, base=base)
    d.T, d.ldy, d.ldbase = (1 << 25) + 1, 1 << 37, 1 << 37
    refused(lambda e: h.adapt([e]), d, "y runs past")
    s = Set(torch, [2, 1], [40, 33], 100, 4, 2, 64)
    d = s.desc()
    d.prefix_len, d.prefix_stride = (1 << 28) + 1, 1 << 35
    refused(h.attend, d, "prefix_k runs past")
    d = s.desc()
    d.n_pages = d.page = 1 << 30
    refused(h.attend, d, "k_pages runs past")
    d = s.desc()
    d.n_tokens, d.q_stride, d.heads, d.kv_heads = (1 << 23) + 1, 1 << 40, 2, 2
    refused(h.attend, d, "q runs past")


def test_sizes_near_32_bits(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 4, 64, 32, 2, 8, torch.bfloat16)
    for name in ("T", "K", "M"):
        d = serving.adapters(x, y, slot, A, B, scale, base=base)
        d.ldx = d.ldy = d.ldbase = d.a_slot = d.b_slot = 1 << 39
        setattr(d, name, (1 << 30) + 1)
        refused(lambda e: h.adapt([e]), d, "out of range")
    d = Set(torch, [2, 1], [40, 33], 100, 1, 1, 64).desc()
    d.n_tokens = (1 << 30) + 1
    refused(h.attend, d, "out of range")
    a = drafts(torch, [2, 1], 64, 1.0, False)
    acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    d = serving.verification(a[0], a[2], a[3], a[4], a[5], acc, tok, q=a[1])
    d.n_drafted = (1 << 30) + 1
    refused(h.verify, d, "out of range")


def test_ranks_of_slots_without_rows(torch, h):
    """R = 0 still reads rank."""
    x, y, slot, A, B, scale, base = make(torch, 4, 64, 32, 2, 0, torch.bfloat16)
    rank = torch.zeros(2, dtype=torch.int32, device="cuda")
    d = serving.adapters(x, y, slot, A, B, scale, rank=rank, base=base)
    d.rank += 2
    refused(lambda e: h.adapt([e]), d, "rank")
