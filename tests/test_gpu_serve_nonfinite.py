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


ROUTES = {  # new, lens, P, H, Hkv, D
    "one split": ([1, 3], [30, 9], 0, 8, 2, 64), "own splits": ([1, 2], [700, 40], 0, 8, 2, 64),
    "prefix by warps": ([1, 2], [37, 20], 500, 8, 2, 128), "prefix alone by warps": ([2], None, 300, 8, 8, 128),
    "tcgen05, one row tile": ([1] * 12, [20] * 12, 900, 4, 1, 128), "tcgen05": ([4] * 20, [20] * 20, 900, 8, 2, 64),
    "tcgen05 alone": ([4] * 20, None, 900, 8, 2, 64)}


def non_finite_where(torch, s, want):
    """Rows the 64-bit form leaves NaN are NaN, the others within the usual tolerance."""
    o = want[0]
    got = s.out.double().cpu()
    bad = torch.isnan(o)
    assert bad.any() and not torch.isfinite(got[bad]).any()
    if not bad.all():
        s.check(torch, want)


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_a_query_of_nan(torch, h, route, dt):
    s = Set(torch, *ROUTES[route], dt=dt)
    s.q[1, 3] = NAN
    s.q[0, 0, 0] = NAN
    h.attend(s.desc())
    torch.cuda.synchronize()
    non_finite_where(torch, s, s.want())


@pytest.mark.parametrize("route", [r for r in ROUTES if ROUTES[r][2]])
@pytest.mark.parametrize("keys", [(0, 128), (130, 131), (256, 300)])
def test_prefix_keys_of_nan(torch, h, route, keys):
    """A whole part of them, and one beside parts that weigh 2^200 times as much."""
    s = Set(torch, *ROUTES[route])
    s.pk[keys[0]:keys[1], 0] = NAN
    h.attend(s.desc())
    torch.cuda.synchronize()
    non_finite_where(torch, s, s.want())
    s = Set(torch, *ROUTES[route], sharp=0.0)
    s.q[:, :, 0] = 8.0
    s.scale = 1.0
    s.pk[:, :, 0] = 0.0
    s.pk[200:220, :, 0] = 20.0
    s.pk[keys[0]:keys[1], 0] = NAN
    h.attend(s.desc())
    torch.cuda.synchronize()
    non_finite_where(torch, s, s.want())


@pytest.mark.parametrize("route", [r for r in ROUTES if ROUTES[r][2]])
@pytest.mark.parametrize("what", [NAN, INF])
def test_prefix_values_that_are_not_finite(torch, h, route, what):
    """Beside keys that weigh 2^200 times as much, too."""
    for heavy in (0.0, 20.0):
        s = Set(torch, *ROUTES[route], sharp=0.0)
        s.q[:, :, 0] = 8.0
        s.scale = 1.0
        s.pk[:, :, 0] = 0.0
        s.pk[200:220, :, 0] = heavy
        s.pv[70, 0, 5] = what
        clean = s.pv.clone()
        clean[70, 0, 5] = 0
        h.attend(s.desc())
        torch.cuda.synchronize()
        got = s.out.double().cpu()
        G = s.q.shape[1] // s.pk.shape[1]
        assert not torch.isfinite(got[:, :G, 5]).any()
        s.pv = clean
        h.attend(s.desc())
        torch.cuda.synchronize()
        keep = torch.ones_like(got, dtype=torch.bool)
        keep[:, :G, 5] = False
        assert torch.equal(got[keep], s.out.double().cpu()[keep])


@pytest.mark.parametrize("route", ROUTES)
def test_scores_of_minus_infinity(torch, h, route):
    """A key whose score is -infinity has no weight; a token with no other key gets zeros; a part that has
    no other key leaves the others as they are, however small their scores."""
    new, lens, P, H, Hkv, D = ROUTES[route]
    for dt in ("bfloat16", "float16"):
        s = Set(torch, *ROUTES[route], dt=dt, sharp=0.0)
        s.q[:, :, 0] = 8.0
        s.scale = 1.0
        for t in (s.pk, s.k):
            if t is not None:
                t[..., 0] = -25.0  # scores of -200
                t[..., 1:] = 0.0
        if P:
            s.pk[:192, :, 0] = -INF
        if lens:
            s.k[s.table[0, 0], ::2, :, 0] = -INF
        want = s.want()
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch, (want[0], want[1], torch.full_like(want[2], 200.0)))
        for t in (s.pk, s.k):
            if t is not None:
                t[..., 0] = -INF
        h.attend(s.desc())
        torch.cuda.synchronize()
        assert (s.out[:int(s.begin[-1])] == 0).all()


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("new", [[1], [1] * 12, [500] * 8])  # parts of few keys and, behind many rows, of many
def test_many_small_weights(torch, h, new, dt):
    """65,535 keys of weight 2^-26 beside one of weight 1 add up to 2^-10.  An f16 weight is rounded to a
    multiple of 2^-24 of its reference, which lies 2^7 below the largest: 2^-32 a key."""
    P = 65536
    s = Set(torch, new, None, P, 8, 1, 64, dt=dt, sharp=0.0)
    s.q[:, :, 0] = 1.0
    s.scale = 1.0
    s.pk.zero_(), s.pv.fill_(1.0)
    s.pk[1:, :, 0] = -18.0
    s.pv[0] = 0.0
    h.attend(s.desc())
    torch.cuda.synchronize()
    crowd = (P - 1) * 2.718281828459045 ** -18
    want = crowd / (1 + crowd)
    got = s.out.double().cpu()
    tol = (0 if dt == "bfloat16" else P * 2.0 ** -32) + (2 * s.u + 2.0 ** -15) * want
    assert (got - want).abs().max() <= tol, (float(got.min()), float(got.max()), want)


@pytest.mark.parametrize("what", [NAN, INF, -INF])
@pytest.mark.parametrize("case", [([6], [50], 40, 4, 2, 64), ([6, 1, 9], [50, 9, 33], 0, 8, 2, 128), ([40], [61], 0, 3, 1, 72),
                                  ([3] * 20, [18] * 20, 300, 4, 1, 128)])
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_later_drafts_that_are_not_finite(torch, h, case, what, dt):
    """What a token may not see does not reach it, in keys and in values."""
    s = Set(torch, *case, dt=dt)
    new, lens = case[0], case[1]
    for b in (0, len(new) - 1):
        j = lens[b] - 1 - new[b] // 2  # one of the new tokens' keys
        at = s.table[b, j // 16]
        s.v[at, j % 16] = what
        want = s.want()
        h.attend(s.desc())
        torch.cuda.synchronize()
        seen = torch.zeros(len(s.q), dtype=torch.bool)
        for c in (0, len(new) - 1)[:1 if b == 0 else 2]:
            t1 = sum(new[:c + 1])
            seen[t1 - new[c] // 2 - 1:t1] = True
        assert not torch.isfinite(s.out.double().cpu()[seen]).any()
        fine = (torch.where(seen.view(-1, 1, 1), torch.full_like(want[0], NAN), want[0]), want[1], want[2])
        s.check(torch, fine)
    j = lens[0] - 1
    s = Set(torch, *case, dt=dt)
    s.k[s.table[0, j // 16], j % 16] = what
    want = s.want()
    want[0][new[0] - 1] = NAN
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, want)


@pytest.mark.parametrize("T", [3, 280])
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_an_infinite_update_beside_a_large_one(torch, h, T, dt):
    x, y, slot, A, B, scale, base = make(torch, T, 64, 32, 1, 2, getattr(torch, dt))
    slot.zero_(), scale.fill_(1.0)
    A.zero_(), B.zero_(), x.zero_()
    A[0, 0, 0], A[0, 1, 1] = INF, 2.0
    x[:, 0], x[:, 1] = 1.0, 60000.0
    x[1, 0] = -1.0
    B[0, :, 0], B[0, :, 1] = 1.0, -1.0
    h.adapt([serving.adapters(x, y, slot, A, B, scale, base=base)])
    torch.cuda.synchronize()
    assert (y[0] == INF).all() and (y[1] == -INF).all()
