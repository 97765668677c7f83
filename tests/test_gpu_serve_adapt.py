"""Handle.adapt: low-rank adapters beside a shared projection, against 64-bit sums.

Tolerance, with u = 2^-23 (the tensor cores truncate their fp32 sums): the base is rounded once when
the update is added; A x is summed in chains of at most K / 256 + 24 additions; B v in chains of at
most 2 R / 8 + 8; v enters with 22 bits."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


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


def close(torch, y, ref, K, R):
    want, s1, s2 = ref
    tol = 2 * U * want.abs() + (K / 256 + 24) * U * s2 + (R / 4 + 12) * U * s1 + 1e-30
    assert not torch.isnan(y).any()
    worst = ((y.double().cpu() - want).abs() / tol).max() if y.numel() else 0
    assert worst <= 1, float(worst)


def make(torch, T, K, M, S, R, dtype, seed=0, off=0, pitch=0):
    """Operands whose rows start `off` elements past a boundary, `pitch` elements longer than they need."""
    g = torch.Generator("cuda").manual_seed(seed)

    def rows(n, m, std, dt, o, extra):
        flat = torch.full((o + n * (m + extra) + 16,), _serve.NAN, dtype=dt, device="cuda")
        v = flat[o:o + n * (m + extra)].view(n, m + extra)[:, :m]
        v.copy_(torch.randn(n, m, device="cuda", generator=g) * std)
        return v

    x = rows(T, K, 1.0, dtype, off, pitch)
    A = torch.as_strided(rows(S, R * K, K ** -0.5 if K else 1.0, dtype, off, pitch), (S, R, K), (R * K + pitch, max(1, K), 1),
                         off)
    B = torch.as_strided(rows(S, M * R, 0.3, dtype, off, pitch), (S, M, R), (M * R + pitch, max(1, R), 1), off)
    base = rows(T, M, 1.0, torch.float32, off, pitch)
    y = rows(T, M, 0.0, torch.float32, off, pitch)
    slot = torch.randint(-1, S, (T,), dtype=torch.int32, device="cuda", generator=g) if S else \
        torch.full((T,), -1, dtype=torch.int32, device="cuda")
    scale = torch.rand(S, device="cuda", generator=g) * 2 - 0.5
    return x, y, slot, A, B, scale, base


SHAPES = [  # T, K, M, S, R
    (1, 64, 32, 1, 4), (1, 4096, 4096, 3, 16), (3, 1, 1, 2, 1), (16, 128, 130, 2, 16), (17, 100, 77, 5, 8),
    (40, 2731, 260, 4, 33), (33, 256, 16, 40, 3), (255, 96, 48, 1, 64), (256, 96, 48, 1, 64), (300, 264, 100, 7, 20),
    (700, 70, 35, 3, 128), (5, 512, 64, 2, 128), (9, 32, 0, 2, 4), (4, 0, 24, 2, 4), (4, 32, 24, 2, 0), (6, 32, 24, 0, 8),
    (0, 32, 24, 2, 8), (2, 40, 40, 4096, 2)]


@pytest.mark.parametrize("T,K,M,S,R", SHAPES)
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("off,pitch", [(0, 0), (1, 3), (8, 8)])
def test_matches_64_bit_sums(torch, h, T, K, M, S, R, dt, off, pitch):
    x, y, slot, A, B, scale, base = make(torch, T, K, M, S, R, getattr(torch, dt), off=off, pitch=pitch)
    rank = torch.tensor([i % (R + 1) for i in range(S)], dtype=torch.int32, device="cuda")
    for rk in (None, rank):
        y.fill_(_serve.NAN)
        h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=rk, base=base)])
        torch.cuda.synchronize()
        close(torch, y, _serve.adapt(x, slot, A, B, scale, rk, base), K, R)


def test_in_place_equals_base_apart(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 50, 200, 90, 4, 16, torch.bfloat16)
    h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
    z = base.contiguous().clone()
    h.adapt([serving.adapters(x, z, slot, A, B, scale)])
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    none = slot < 0
    assert none.any() and torch.equal(z[none], base[none])


def test_what_lies_past_a_rank_is_not_used(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 20, 128, 64, 3, 24, torch.float16)
    rank = torch.tensor([5, 0, 16], dtype=torch.int32, device="cuda")
    h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=rank, base=base)])
    first = y.clone()
    for s, r in enumerate([5, 0, 16]):
        A[s, r:], B[s, :, r:] = _serve.NAN, _serve.INF
    y.fill_(_serve.NAN)
    h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=rank, base=base)])
    torch.cuda.synchronize()
    assert torch.equal(first, y)


def test_a_token_does_not_depend_on_its_batch(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 60, 300, 120, 4, 32, torch.bfloat16)
    h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
    one = torch.full_like(y, _serve.NAN)
    for t in range(60):
        h.adapt([serving.adapters(x[t:t + 1], one[t:t + 1], slot[t:t + 1], A, B, scale, base=base[t:t + 1])])
    torch.cuda.synchronize()
    assert torch.equal(one, y)


def test_many_projections_in_one_call(torch, h):
    sets = [make(torch, 12, 64 + 8 * i, 40 + i, 3, 1 + 3 * i, torch.bfloat16 if i % 3 else torch.float16, seed=i)
            for i in range(19)]
    before = h.kernel_launches()
    h.adapt([serving.adapters(x, y, s, A, B, c, base=b) for x, y, s, A, B, c, b in sets])
    torch.cuda.synchronize()
    assert h.kernel_launches() > before
    for x, y, s, A, B, c, b in sets:
        close(torch, y, _serve.adapt(x, s, A, B, c, None, b), x.shape[1], A.shape[1])
    h.adapt([])


def test_zero_base_and_infinite_inputs(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 8, 64, 32, 2, 8, torch.bfloat16)
    d = serving.adapters(x, y, slot, A, B, scale, base=base)
    d.base = None
    h.adapt([d])
    torch.cuda.synchronize()
    close(torch, y, _serve.adapt(x, slot, A, B, scale, None, torch.zeros_like(base)), 64, 8)
    A.zero_(), B.zero_()
    A[:, 0, 0], B[:, 0, 0], x[0, 0] = 1.0, 1.0, _serve.INF
    slot.fill_(0)
    scale.fill_(1.0)
    one = torch.ones(2, dtype=torch.int32, device="cuda")  # the other ranks would add 0 * infinity
    h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=one, base=base)])
    torch.cuda.synchronize()
    assert y[0, 0] == _serve.INF and torch.isfinite(y[1:]).all()


def test_slots_and_ranks_outside_the_descriptor(torch):
    with wt.Handle([]) as h:
        x, y, slot, A, B, scale, base = make(torch, 9, 64, 32, 2, 8, torch.bfloat16)
        slot[:] = torch.tensor([0, 1, 2, 99, -5, 2 ** 31 - 1, 0, 1, -2 ** 31], dtype=torch.int32)
        h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
        torch.cuda.synchronize()
        close(torch, y, _serve.adapt(x, slot, A, B, scale, None, base), 64, 8)
        assert h.device_status() == wt.WT_EINVAL
    with wt.Handle([]) as h:
        rank = torch.tensor([-3, 1000], dtype=torch.int32, device="cuda")
        h.adapt([serving.adapters(x, y, slot, A, B, scale, rank=rank, base=base)])
        torch.cuda.synchronize()
        close(torch, y, _serve.adapt(x, slot, A, B, scale, rank, base), 64, 8)
        assert h.device_status() == wt.WT_EINVAL


def test_other_streams_and_graphs(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 33, 256, 96, 3, 16, torch.float16)
    want = _serve.adapt(x, slot, A, B, scale, None, base)
    d = [serving.adapters(x, y, slot, A, B, scale, base=base)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h.adapt(d, s.cuda_stream)
    s.synchronize()
    close(torch, y, want, 256, 16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.adapt(d, torch.cuda.current_stream().cuda_stream)
    y.fill_(_serve.NAN)
    slot.copy_(slot.flip(0).clone())  # a replay reads the slots of its own time
    g.replay()
    torch.cuda.synchronize()
    close(torch, y, _serve.adapt(x, slot, A, B, scale, None, base), 256, 16)


def test_refusals(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 4, 64, 32, 2, 8, torch.bfloat16)

    def refused(code=wt.WT_EINVAL, **change):
        d = serving.adapters(x, y, slot, A, B, scale, base=base)
        for k, v in change.items():
            setattr(d, k, v)
        with pytest.raises(wt.WtError) as e:
            h.adapt([d])
        assert e.value.code == code and "wt_adapt" in str(e.value)

    for name in ("x", "y", "slot", "A", "B"):
        refused(**{name: None})
    refused(wt.WT_ENOTSUP, dtype=wt.WT_F32)
    refused(wt.WT_ENOTSUP, dtype=wt.WT_I8)
    refused(dtype=17)
    for name in ("T", "K", "M", "S", "R"):
        refused(**{name: -1})
    refused(R=129), refused(S=4097), refused(ldx=63), refused(ldy=31), refused(ldbase=31)
    refused(a_slot=8 * 64 - 1), refused(b_slot=8 * 32 - 1), refused(ldx=1 << 41)
    refused(x=x.data_ptr() + 1), refused(y=y.data_ptr() + 2)
    refused(base=y.data_ptr() + 4), refused(base=y.data_ptr(), ldbase=33)
    refused(T=1 << 30), refused(ldy=1 << 39)  # runs past the allocation
    with pytest.raises(ValueError):
        serving.adapters(x.float(), y, slot, A, B)
    with pytest.raises(ValueError):
        serving.adapters(x, y, slot.long(), A, B)
    with pytest.raises(ValueError):
        serving.adapters(x, y, slot, A, B[:, :-1])
    with pytest.raises(ValueError):
        serving.adapters(x, y, slot, A, B, base=base[:1].expand(4, 32))
    with pytest.raises(ValueError):
        serving.adapters(x.cpu(), y, slot, A, B)


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("R", [4, 10, 12, 16, 20, 24, 40, 72, 100])
def test_ranks_off_the_vectors(torch, h, T, R):
    """Rows of B whose length is no multiple of a 16-byte vector, in both forms."""
    x, y, slot, A, B, scale, base = make(torch, T, 72, 150, 4, R, torch.float16)
    h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
    torch.cuda.synchronize()
    close(torch, y, _serve.adapt(x, slot, A, B, scale, None, base), 72, R)


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_updates_of_any_size(torch, h, dt):
    """Tokens whose A x lies far apart, in one launch of many tokens."""
    x, y, slot, A, B, scale, base = make(torch, 280, 64, 96, 2, 16, getattr(torch, dt))
    slot.clamp_(min=0)
    size = 10.0 ** (torch.arange(280, device="cuda") % 9 - 4.0)
    x.copy_(x.float() * size.view(-1, 1))
    x[7] = 0
    base.zero_()
    h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
    torch.cuda.synchronize()
    close(torch, y, _serve.adapt(x, slot, A, B, scale, None, base), 64, 16)


@pytest.mark.parametrize("T", [3, 260])
def test_offsets_past_32_bits(torch, h, T):
    x, y, slot, A, B, scale, base = make(torch, T, 64, 32, 2, 8, torch.bfloat16)
    far = torch.empty((1 << 31) + 8 * 64, dtype=torch.bfloat16, device="cuda")
    A2 = far.as_strided((2, 8, 64), (1 << 31, 64, 1))
    A2.copy_(A)
    big = torch.empty((1 << 31) + 32 * T, device="cuda")
    y2 = big[-32 * T:].view(T, 32) if T > 3 else big.as_strided((3, 32), (1 << 30, 1))
    h.adapt([serving.adapters(x, y2, slot, A2, B, scale, base=base)])
    torch.cuda.synchronize()
    close(torch, y2, _serve.adapt(x, slot, A, B, scale, None, base), 64, 8)
