"""Handle.attend: a shared prefix and paged caches of each request, against 64-bit attention.

Tolerance, with u the unit roundoff of the caches' type (2^-8 bf16, 2^-11 f16): the weights p are
rounded once to that type (u of sum p |v|; an f16 weight below 2^-14 by up to 2^-25), the output
once (u of |o|); a score is a sum in fp32 truncated at each of at most head_dim / 16 + 4 steps
(2^-23 of sum |q| |k| each), which moves every p by that much relative; the sums of p and p v and
the joining of parts add 2^-15."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve

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


class Set:
    """Inputs of one call: `new` and `lens` per request."""

    def __init__(self, torch, new, lens, P, H, Hkv, D, page=16, dt="bfloat16", seed=0, fused=0, sharp=1.0, head_major=False):
        g = torch.Generator("cuda").manual_seed(seed)
        dt = getattr(torch, dt)
        self.u = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -11

        def normal(*shape):
            return torch.randn(shape, device="cuda", generator=g).to(dt)

        N, B = sum(new), len(new)
        self.begin = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
        self.q = (normal(N, H + fused, D) * sharp)[:, :H]
        self.out = torch.full((N, H + fused, D), _serve.NAN, dtype=dt, device="cuda")[:, :H]
        self.pk = self.pv = None
        if P:
            self.pk, self.pv = (normal(Hkv, P, D).transpose(0, 1) if head_major else normal(P, Hkv, D) for _ in range(2))
        self.k = self.v = self.table = self.lens = None
        self.max_new, self.max_len, self.scale = max(new), 0, D ** -0.5
        if lens is not None:
            self.max_len = max(lens)
            pages = [-(-n // page) for n in lens]
            total, most = sum(pages) + 2, max(max(pages), 1)
            order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
            table = torch.full((B, most), -1, dtype=torch.int32)
            self.k, self.v = (torch.full((total, page, Hkv, D), _serve.NAN, dtype=dt, device="cuda") for _ in range(2))
            self.v[::2] = _serve.INF
            for b, n in enumerate(lens):
                for i in range(pages[b]):
                    at = order.pop()
                    table[b, i] = at
                    m = min(page, n - i * page)
                    self.k[at, :m], self.v[at, :m] = normal(m, Hkv, D), normal(m, Hkv, D)
            self.table, self.lens = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")

    def desc(self, **more):
        return serving.attention(self.q, self.out, self.begin, self.k, self.v, self.table, self.lens,
                                 **{**dict(max_new=self.max_new, max_len=self.max_len, prefix_k=self.pk, prefix_v=self.pv,
                                           scale=self.scale), **more})

    def want(self):
        return _serve.attend(self.q, self.begin, self.pk, self.pv, self.k, self.v, self.table, self.lens, self.scale)

    def check(self, torch, want=None):
        o, mag, qk = want or self.want()
        keys = (0 if self.pk is None else len(self.pk)) + self.max_len
        vmax = max([float(t.abs()[torch.isfinite(t)].max()) for t in (self.pv, self.v) if t is not None and t.numel()] + [0.0])
        D = self.q.shape[2]
        small = keys * 2.0 ** -25 * vmax if self.u == 2.0 ** -11 else 0.0
        tol = (self.u + 2 * (D / 16 + 4) * 2.0 ** -23 * qk + 2.0 ** -15) * mag + self.u * o.abs() + small + 1e-30
        got = self.out.double().cpu()
        rows = ~torch.isnan(o)
        assert rows.any() or o.numel() == 0
        worst = ((got - o).abs() / tol)[rows]
        assert not torch.isnan(got[rows]).any() and (worst.numel() == 0 or worst.max() <= 1), float(worst.max())


CASES = [  # new, lens, P, H, Hkv, D, page
    ([1], [1], 0, 1, 1, 8, 16), ([1], None, 1, 4, 4, 64, 1), ([1], None, 500, 32, 8, 128, 1), ([1], [37], 500, 32, 8, 128, 16),
    ([1], [700], 0, 8, 8, 128, 1), ([2, 3], [2, 3], 0, 4, 2, 72, 7), ([1, 1, 1], [5, 64, 129], 64, 8, 1, 96, 64),
    ([3, 1, 4, 2], [3, 50, 33, 300], 257, 12, 4, 80, 24), ([5, 8], [20, 8], 130, 16, 2, 128, 16), ([16], [100], 1000, 8, 2, 128, 32),
    ([1] * 40, [7 + i for i in range(40)], 300, 8, 2, 64, 16), ([2] * 20, None, 777, 6, 2, 40, 1), ([7], [1000], 3, 128, 1, 56, 128),
    ([1, 2], [300, 2], 2049, 5, 5, 104, 48), ([33], [90], 200, 3, 1, 128, 16), ([130], [130], 0, 2, 1, 64, 16),
    ([4] * 33, [40] * 33, 1500, 4, 1, 128, 16)]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_matches_64_bit_attention(torch, h, case, dt):
    new, lens, P, H, Hkv, D, page = case
    s = Set(torch, new, lens, P, H, Hkv, D, page, dt, fused=len(new) % 3, head_major=P % 2 == 1)
    want = s.want()
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, want)
    if s.out.shape[0] > 1 and len(new) % 3:  # what lies between the tokens' heads is not written
        assert torch.isnan(torch.as_strided(s.out, (s.out.shape[0], s.out.stride(0)), (s.out.stride(0), 1))[:-1, H * D:]).all()


def test_sharp_scores_and_large_values(torch, h):
    for sharp in (30.0, 1e-3):
        s = Set(torch, [2, 1], [40, 300], 900, 8, 2, 128, dt="float16", sharp=sharp)
        s.pv *= 100
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch)
    for scale in (0.0, -0.2, 5.0):
        s = Set(torch, [2, 1], [40, 300], 900, 8, 2, 128)
        s.scale = scale
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch)


def test_scores_that_grow_along_the_keys(torch, h):
    """Each tile raises the row's maximum, so every partial sum is rescaled."""
    s = Set(torch, [1] * 36, [200] * 36, 3001, 4, 1, 128, sharp=0.0)
    s.q[:, :, 0] = 8.0
    s.pk[:, :, 0] = torch.linspace(-60, 60, 3001, device="cuda").to(s.pk.dtype).view(-1, 1)
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)
    s.pk[:, :, 0] = s.pk[:, :, 0].flip(0)
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)


def test_tokens_without_keys_are_zero(torch, h):
    # fewer own keys than new tokens: the first ones see nothing
    s = Set(torch, [4, 2, 3], [2, 0, 3], 0, 4, 2, 64)
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)
    assert (s.out[:2] == 0).all() and (s.out[4:6] == 0).all() and (s.out[2:4] != 0).any()
    s = Set(torch, [2, 1], None, 0, 4, 4, 64)
    h.attend(s.desc())
    torch.cuda.synchronize()
    assert (s.out == 0).all()
    s = Set(torch, [3, 1], [1, 0], 70, 4, 2, 64)  # the prefix is still there
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)


def test_requests_without_new_tokens_and_spare_rows(torch, h):
    s = Set(torch, [0, 3, 0, 1], [9, 30, 0, 17], 100, 4, 2, 64)
    h.attend(s.desc(max_new=8, max_len=s.table.shape[1] * 16))
    torch.cuda.synchronize()
    s.check(torch)
    # rows past the last request's are left alone
    s = Set(torch, [2, 2], [9, 30], 100, 4, 2, 64)
    s.begin[2] = 3
    want = s.want()
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, want)
    assert torch.isnan(s.out[3]).all()


def test_a_token_does_not_see_later_drafts(torch, h):
    s = Set(torch, [6], [50], 40, 4, 2, 64)
    h.attend(s.desc())
    first = s.out.clone()
    for j in range(45, 50):
        at = s.table[0, j // 16]
        s.k[at, j % 16], s.v[at, j % 16] = 3.0, -5.0
        h.attend(s.desc())
        torch.cuda.synchronize()
        seen = j - 44
        assert torch.equal(s.out[:seen], first[:seen]) or j > 45
        s.check(torch)


def test_streams_graphs_and_workspaces(torch, h):
    a = Set(torch, [1] * 8, [60] * 8, 2000, 8, 2, 128, seed=1)
    b = Set(torch, [2] * 3, [33] * 3, 500, 8, 2, 128, seed=2)
    wa, wb = a.want(), b.want()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (sa, sb):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        h.attend(a.desc(), sa.cuda_stream)
        h.attend(b.desc(), sb.cuda_stream)
    torch.cuda.synchronize()
    a.check(torch, wa), b.check(torch, wb)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st = torch.cuda.current_stream().cuda_stream
        h.attend(a.desc(), st)
        h.attend(b.desc(), st)
    a.q.copy_(a.q.flip(0).clone())
    wa = a.want()
    a.out.fill_(_serve.NAN), b.out.fill_(_serve.NAN)
    for _ in range(3):
        g.replay()
        h.attend(b.desc(), sb.cuda_stream)
    torch.cuda.synchronize()
    a.check(torch, wa), b.check(torch, wb)
    for _ in range(12):  # more streams than the handle keeps workspaces for
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        h.attend(a.desc(), s.cuda_stream)
    torch.cuda.synchronize()
    a.check(torch, wa)


def test_close_returns_the_workspaces(torch):
    before = wt.live()
    s = Set(torch, [1] * 8, [60] * 8, 2000, 8, 2, 128)
    for _ in range(3):
        with wt.Handle([]) as h:
            h.attend(s.desc())
            torch.cuda.synchronize()
    after = wt.live()
    assert {k: after[k] for k in ("handles", "events", "device_bytes")} == {k: before[k] for k in ("handles", "events", "device_bytes")}


def test_an_allocation_that_fails(torch, h, monkeypatch):
    s = Set(torch, [1], [60], 2000, 8, 2, 128)
    monkeypatch.setenv("WT_FAULT", "alloc")
    with pytest.raises(wt.WtError) as e:
        h.attend(s.desc())
    assert e.value.code == wt.WT_ENOMEM
    monkeypatch.delenv("WT_FAULT")
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)


def test_values_outside_the_descriptor(torch):
    def status(s, **more):
        with wt.Handle([]) as h:
            h.attend(s.desc(**more))
            torch.cuda.synchronize()
            return h.device_status()

    s = Set(torch, [2, 1], [40, 33], 100, 4, 2, 64)
    keep = s.table.clone()
    for bad in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):  # a page that is not there: its keys are absent
        s.table.copy_(keep)
        s.table[0, 0] = bad
        assert status(s) == wt.WT_EINVAL
    s.table.copy_(keep)
    left = Set(torch, [2, 1], [24, 33], 100, 4, 2, 64)
    for a, b in (("q", "q"), ("pk", "pk"), ("pv", "pv")):
        getattr(left, a).copy_(getattr(s, b))
    left.k, left.v, left.table = s.k, s.v, torch.stack([s.table[0].roll(-1), s.table[1]]).contiguous()
    s.table[0, 0] = -1
    assert status(s) == wt.WT_EINVAL
    s.check(torch, left.want())
    s.table.copy_(keep)
    for bad in ([0, 9, 3], [-4, 2, 3], [2, 0, 3], [0, 2, 2 ** 31 - 1]):
        s.begin.copy_(torch.tensor(bad, dtype=torch.int32))
        assert status(s) == wt.WT_EINVAL
    s.begin.copy_(torch.tensor([0, 2, 3], dtype=torch.int32))
    for bad in ([-1, 33], [10 ** 9, 33]):
        s.lens.copy_(torch.tensor(bad, dtype=torch.int32))
        assert status(s) == wt.WT_EINVAL
    s.lens.copy_(torch.tensor([40, 33], dtype=torch.int32))
    assert status(s) == 0
    s.check(torch)


def test_refusals(torch, h):
    s = Set(torch, [2, 1], [40, 33], 100, 4, 2, 64)

    def refused(code=wt.WT_EINVAL, **change):
        d = s.desc()
        for k, v in change.items():
            setattr(d, k, v)
        with pytest.raises(wt.WtError) as e:
            h.attend(d)
        assert e.value.code == code and "wt_attend" in str(e.value)

    for name in ("q", "out", "begin", "prefix_k", "prefix_v", "k_pages", "v_pages", "table", "len"):
        refused(**{name: None})
    refused(wt.WT_ENOTSUP, dtype=wt.WT_F32), refused(dtype=-2), refused(wt.WT_ENOTSUP, head_dim=136), refused(head_dim=12)
    refused(head_dim=0), refused(kv_heads=3), refused(kv_heads=0), refused(heads=0), refused(n_req=-1), refused(n_req=70000)
    refused(n_tokens=-1), refused(max_new=-1), refused(prefix_len=-1), refused(max_len=-1), refused(page=0)
    refused(max_len=10 ** 6), refused(n_pages=10 ** 8), refused(n_tokens=10 ** 8), refused(prefix_len=10 ** 8)
    refused(q_stride=248), refused(q_stride=260), refused(out_stride=0), refused(prefix_stride=60), refused(prefix_head=63)
    refused(q=s.q.data_ptr() + 2), refused(prefix_k=s.pk.data_ptr() + 8), refused(table_stride=-1)
    refused(scale=float("nan")), refused(scale=float("inf"))
    for bad in (dict(max_len=10 ** 5), dict(prefix_v=None), dict(prefix_v=s.pv[:-1]), dict(prefix_k=s.pk.float())):
        with pytest.raises(ValueError):
            s.desc(**bad)
    with pytest.raises(ValueError):
        serving.attention(s.q, s.out[:, :2], s.begin, max_new=2)


@pytest.mark.parametrize("P", [1, 5, 100, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("G,D", [(1, 128), (4, 64), (5, 96), (128, 128)])
def test_batches_behind_short_prefixes(torch, h, P, G, D):
    """Many rows, few keys: key tiles and row tiles that are hardly filled."""
    new = [2, 0, 3, 1] * (12 if G < 128 else 1)
    s = Set(torch, new, [n + 3 for n in new], P, 2 * G, 2, D, seed=P)
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)


@pytest.mark.parametrize("P,H,D,dt", [(100, 160, 8, "bfloat16"), (300, 160, 64, "float16"), (1595, 20, 128, "float16"),
                                     (1595, 40, 128, "bfloat16"), (600, 75, 72, "bfloat16")])
def test_ranges_of_few_tiles_over_many_heads(torch, h, P, H, D, dt):
    """One row tile, and ranges of key tiles that meet several heads with one tile of some of them: the
    stream of the odd tiles then has none, and must not run ahead of the stream of the even ones."""
    s = Set(torch, [2] * 20, [12] * 20, P, H, H, D, dt=dt)
    want = s.want()
    for _ in range(20):
        s.out.fill_(_serve.NAN)
        h.attend(s.desc())
        torch.cuda.synchronize()
        s.check(torch, want)


@pytest.mark.parametrize("scale", [0.3, -0.3, 0.0])
def test_batches_at_any_scale(torch, h, scale):
    s = Set(torch, [3] * 16, [20] * 16, 300, 8, 2, 64)
    s.scale = scale
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch)


def test_offsets_past_32_bits(torch, h):
    """A pool of more than 2^31 elements, and a prefix whose keys lie as far apart."""
    s = Set(torch, [1, 2], [40, 33], 3, 4, 2, 128)
    total = (1 << 31) // (16 * 2 * 128) + 40
    k, v = (torch.empty(total, 16, 2, 128, dtype=s.k.dtype, device="cuda") for _ in range(2))
    far = s.k.shape[0]
    k[-far:], v[-far:] = s.k, s.v
    s.k, s.v = k, v
    s.table += total - far
    pk, pv = (torch.empty((1 << 31) + 4096, dtype=k.dtype, device="cuda").as_strided((3, 2, 128), (1 << 30, 128, 1))
              for _ in range(2))
    pk.copy_(s.pk), pv.copy_(s.pv)
    s.pk, s.pv = pk, pv
    near = Set(torch, [1, 2], [40, 33], 3, 4, 2, 128)
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, near.want())


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("rise", [0.0, 1.3, 5.2])
def test_roundings_that_weights_share_cancel(torch, h, dt, rise):
    """Scores of two kinds, so that most weights are one number and share its rounding: it must not show in
    the result, which then errs to both sides alike (128 columns and more: a mean error of 0.2 u would be
    four standard deviations of roundings alone)."""
    for new in ([1, 2], [2] * 20):  # on the warp kernel and on tcgen05
        s = Set(torch, new, [40] * len(new), 4000, 4, 2, 128, dt=dt, sharp=0.0)
        s.q[:, :, 0] = 1.0
        s.scale = 1.0
        s.pk[:, :, 0] = rise * (torch.arange(4000, device="cuda") // 128 % 2).view(-1, 1).to(s.pk.dtype)
        s.k[:, :, :, 0] = 0.0
        for v in (s.pv, s.v):
            v += torch.linspace(1, 8, 128, device="cuda").to(v.dtype)
        h.attend(s.desc())
        torch.cuda.synchronize()
        o, _, _ = s.want()
        off = (s.out.double().cpu() - o) / o
        assert off.abs().max() <= 1.1 * s.u and off.mean().abs() <= 0.2 * s.u
