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


def test_overlapping_buffers_are_refused(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 4, 64, 32, 2, 8, torch.bfloat16)
    rank = torch.full((2,), 8, dtype=torch.int32, device="cuda")

    def adapt(**change):
        d = serving.adapters(x, y, slot, A, B, scale, rank=rank, base=base)
        for k, v in change.items():
            setattr(d, k, v)
        return d

    one = lambda d: h.adapt([d])  # noqa: E731
    big = torch.zeros(1 << 16, device="cuda")
    at = big.data_ptr()
    for name in ("x", "A", "B", "slot", "rank", "scale", "base"):
        refused(one, adapt(y=at, ldy=32, **{name: at + 256}), "overlap")
    refused(one, adapt(base=y.data_ptr() + 16), "overlap")
    for name in ("x", "A", "B", "slot", "rank", "scale", "base"):
        d = adapt(**{name: at + 256})
        other = adapt(y=at, ldy=32)
        refused(h.adapt, [d, other], "overlap"), refused(h.adapt, [other, d], "overlap")
    refused(h.adapt, [adapt(y=at, ldy=32), adapt(y=at + 64, ldy=40)], "overlap")

    s = Set(torch, [2, 1], [40, 33], 100, 4, 2, 64)
    n = s.out.numel() * 2
    for name in ("q", "begin", "prefix_k", "prefix_v", "k_pages", "v_pages", "table", "len"):
        d = s.desc()
        setattr(d, name, at + n - 16)
        d.out = at
        refused(h.attend, d, "overlap")
    d = s.desc()
    d.out, d.out_stride = d.q, d.q_stride + 8
    refused(h.attend, d, "overlap")

    l, p = torch.randn(3, 64, device="cuda"), torch.empty(3, 64, device="cuda")
    t = torch.ones(3, device="cuda")
    d = serving.probabilities(l, p, temperature=t)
    d.temp = p.data_ptr() + 4
    refused(h.probs, d, "overlap")

    a = drafts(torch, [2, 1], 64, 1.0, False)
    acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")

    def verify(**change):
        d = serving.verification(a[0], a[2], a[3], a[4], a[5], acc, tok, q=a[1])
        for k, v in change.items():
            setattr(d, k, v)
        return d

    for name in ("p", "q", "drafted", "begin", "u", "u_draw", "accepted"):
        refused(h.verify, verify(tokens=at, **{name: at + 4}), "overlap")
    for name in ("p", "q", "drafted", "begin", "u", "u_draw"):
        refused(h.verify, verify(accepted=at, **{name: at + 4}), "overlap")


def test_buffers_that_interleave_are_accepted(torch, h):
    """Columns of one buffer, as fused projections and gathered outputs leave them."""
    x, y, slot, A, B, scale, base = make(torch, 40, 64, 32, 2, 8, torch.bfloat16)
    one = torch.full((40, 100), _serve.NAN, device="cuda")
    one[:, 32:64] = base
    want = _serve.adapt(x, slot, A, B, scale, None, base)
    h.adapt([serving.adapters(x, one[:, :32], slot, A, B, scale, base=one[:, 32:64]),
             serving.adapters(x, one[:, 64:96], slot, A, B, scale, base=one[:, 32:64])])
    torch.cuda.synchronize()
    close(torch, one[:, :32], want, 64, 8), close(torch, one[:, 64:96], want, 64, 8)
    assert torch.isnan(one[:, 96:]).all()
    # rows of other pitches between one another's: y in the gaps of every second row of base
    wide = torch.full((80, 100), _serve.NAN, device="cuda")
    pairs = wide.view(40, 200)
    pairs[:, 140:172] = base
    h.adapt([serving.adapters(x, wide[:40, :32], slot, A, B, scale, base=pairs[:, 140:172])])
    torch.cuda.synchronize()
    close(torch, wide[:40, :32], want, 64, 8)

    l = torch.randn(9, 1003, device="cuda")
    both = torch.full((9, 2100), _serve.NAN, device="cuda")
    both[:, 1050:2053] = l
    h.probs(serving.probabilities(both[:, 1050:2053], both[:, 3:1006]))
    torch.cuda.synchronize()
    want = torch.softmax(l.double(), dim=1)
    assert ((both[:, 3:1006].double() - want).abs() <= 1e-5 * want + 1e-12).all()

    for new, lens, P in (([2, 1], [40, 33], 0), ([2, 1], [40, 33], 100), ([2] * 20, [9] * 20, 300)):
        s = Set(torch, new, lens, P, 4, 2, 64)
        want = s.want()
        fused = torch.cat([s.q, torch.full_like(s.q, _serve.NAN)], dim=1)
        s.q, s.out = fused[:, :4], fused[:, 4:]
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch, want)
        s.out = s.q  # in place
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch, want)


def test_a_table_that_is_part_of_a_wider_one(torch, h):
    """Its last row ends with its allocation."""
    torch.cuda.empty_cache()
    s = Set(torch, [2, 1], [40, 33], 100, 4, 2, 64)
    wide = torch.full((8, 1 << 20), -1, dtype=torch.int32, device="cuda")  # a 32 MB allocation of its own
    part = wide[6:, (1 << 20) - s.table.shape[1]:]
    part.copy_(s.table)
    want = s.want()
    s.table = part
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, want)


def test_strides_of_dimensions_of_one(torch, h):
    """They say nothing: two prefixes that differ in them alone are alike."""
    for P, Hkv in ((1, 2), (60, 1), (1, 1)):
        s = Set(torch, [2, 1], [40, 33], P, 4, Hkv, 64)
        want = s.want()
        st = list(s.pv.stride())
        if P == 1:
            st[0] = 8 * 64 * Hkv
        if Hkv == 1:
            st[1] = 8 * 64
        s.pv = torch.as_strided(s.pv, s.pv.shape, st)
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch, want)


@pytest.mark.parametrize("new", [[2, 1], [2] * 30])
@pytest.mark.parametrize("P", [0, 100])
def test_offsets_that_contradict_a_call_without_own_keys(torch, new, P):
    """On the warp kernel, on tcgen05 and with no key at all."""
    B, n = len(new), sum(new)
    for at, bad in ((1, 9), (0, -4), (B, 2 ** 31 - 1), (1, -2 ** 31)):
        s = Set(torch, new, None, P, 4, 2, 64)
        s.begin[at] = bad
        with wt.Handle([]) as h:
            h.attend(s.desc())
            torch.cuda.synchronize()
            assert h.device_status() == wt.WT_EINVAL
    s = Set(torch, new, None, P, 4, 2, 64)
    with wt.Handle([]) as h:
        h.attend(s.desc())
        torch.cuda.synchronize()
        assert h.device_status() == 0
