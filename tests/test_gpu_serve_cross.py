"""wt_cross against 64 bits: memories of any length, states left out, heads, strides, and rows that see nothing."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve_more as plain

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


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
    """Requests of `new` tokens and memories of `mem` states, laid out one after another with gaps of NaN and
    infinity between them."""

    def __init__(self, torch, new, mem, H, Hkv, D, dt="bfloat16", holes=None, layout="states", sharp=1.0, gap=3, pad=0, between=0, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        dt = getattr(torch, dt)
        self.u = torch.finfo(dt).eps / 2

        def normal(*shape):
            return torch.randn(shape, device="cuda", generator=g).to(dt)

        def ints(v):
            return torch.tensor(v, dtype=torch.int32, device="cuda")

        N = sum(new) + pad
        self.begin = ints([sum(new[:b]) for b in range(len(new) + 1)])
        self.q = (normal(N, H + between, D) * sharp)[:, :H]
        self.out = torch.full((N, H + between, D), NAN, dtype=dt, device="cuda")[:, :H]
        at, starts = 0, []
        for n in mem:
            at += gap
            starts.append(at)
            at += n
        M = at + gap
        if layout == "states":
            self.k, self.v = normal(M, Hkv, D), normal(M, Hkv, D)
        elif layout == "heads":
            self.k, self.v = normal(Hkv, M, D).transpose(0, 1), normal(Hkv, M, D).transpose(0, 1)
        else:
            self.k, self.v = normal(M, 2, Hkv, D).unbind(dim=1)
        inside = torch.zeros(M, dtype=torch.bool, device="cuda")
        for s, n in zip(starts, mem):
            inside[s:s + n] = True
        self.keep = None
        if holes is not None:
            self.keep = ((torch.rand(M, device="cuda", generator=g) >= holes) & inside).to(torch.uint8)
            self.keep[::7] *= 200  # anything but 0 keeps
            inside &= self.keep != 0
        self.k[~inside], self.v[~inside] = NAN, INF
        self.inside = inside
        self.mem_begin, self.mem_len = ints(starts), ints(mem)
        self.max_new, self.max_mem, self.scale = max(new), max(mem), D ** -0.5

    def desc(self, **kw):
        return serving.cross_attention(self.q, self.out, self.begin, self.k, self.v, self.mem_begin, self.mem_len,
                                       **{**dict(max_new=self.max_new, max_mem=self.max_mem, keep=self.keep, scale=self.scale), **kw})

    def want(self):
        return plain.cross(self.q, self.begin, self.k, self.v, self.mem_begin, self.mem_len, self.keep, self.scale)

    def check(self, torch, want=None):
        """The weights' rounding and the output's: u each (of sum p |v| and of the result); scores: D / 16 + 4 sums in
        fp32 of up to sum |q k|, twice (score and maximum); sums of weights and values: 2^-15.  f16 weights below
        2^-32 of the largest may vanish."""
        o, mag, qk = want or self.want()
        D = self.q.shape[2]
        vmax = float(self.v.abs()[torch.isfinite(self.v)].max()) if torch.isfinite(self.v).any() else 0.0
        small = self.max_mem * 2.0 ** -25 * vmax if self.u == 2.0 ** -11 else 0.0
        tol = (self.u + 2 * (D / 16 + 4) * 2.0 ** -23 * qk + 2.0 ** -15) * mag + self.u * o.abs() + small + 1e-30
        got = self.out.double().cpu()
        rows = ~torch.isnan(o)
        worst = ((got - o).abs() / tol)[rows]
        assert not torch.isnan(got[rows]).any() and (worst.numel() == 0 or worst.max() <= 1), float(worst.max())


# new, mem, H, Hkv, D
CASES = [([1], [1], 1, 1, 8), ([1], [16], 2, 1, 64), ([1], [63], 4, 4, 72), ([1], [64], 4, 4, 64), ([1], [65], 4, 2, 128),
         ([1], [1500], 32, 8, 128), ([1], [5000], 16, 1, 128), ([1, 1, 1], [5, 0, 129], 8, 1, 96), ([2, 0, 3], [20, 9, 333], 4, 2, 80),
         ([1] * 40, [7 + 31 * i for i in range(40)], 4, 4, 64), ([5, 3], [700, 41], 8, 8, 80), ([4] * 9, [300] * 9, 12, 4, 40),
         ([7], [129], 128, 1, 56), ([8, 8], [128, 256], 8, 2, 128), ([33], [90], 3, 1, 128), ([16, 40], [127, 300], 4, 1, 64),
         ([130], [130], 2, 1, 64), ([257, 1, 100], [1000, 77, 300], 2, 2, 64), ([300], [640], 4, 1, 128), ([200, 150], [385, 511], 5, 5, 104),
         ([70, 129, 64], [1, 128, 129], 6, 2, 72), ([513], [2000], 2, 1, 96), ([65] * 12, [100 + 90 * i for i in range(12)], 4, 2, 128),
         ([9, 200], [300, 40], 24, 8, 88), ([100], [333], 3, 3, 16), ([48, 47], [200, 1300], 20, 20, 64), ([3, 129], [900, 900], 128, 1, 128),
         ([77, 5], [400, 260], 65, 1, 24)]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
@pytest.mark.parametrize("holes", [None, 0.4])
def test_matches_64_bits(torch, h, case, dt, holes):
    new, mem, H, Hkv, D = CASES[case]
    s = Set(torch, new, mem, H, Hkv, D, dt, holes, layout=("states", "heads", "fused")[case % 3], between=case % 2, pad=case % 4, seed=case)
    h.cross(s.desc())
    s.check(torch)
    N = sum(new)
    assert torch.isnan(s.out[N:]).all()  # rows that no request holds
    if case % 2 and len(s.out) > 1:  # what lies between the tokens' heads
        whole = torch.as_strided(s.out, (len(s.out), s.out.stride(0)), (s.out.stride(0), 1))
        assert torch.isnan(whole[:-1, H * D:]).all()


ROUTES = {"few": ([1, 3, 1], [300, 1000, 0], 8, 2, 64), "one row tile": ([30, 9, 25], [300, 1000, 0], 8, 2, 128),
          "many": ([300, 70, 64], [500, 1000, 0], 8, 4, 64)}


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_masks_that_leave_little(torch, h, route, dt):
    """Memories of which one state is kept, the first, the last or none; and almost none of all."""
    s = Set(torch, *ROUTES[route], dt=dt, holes=0.97)
    m0 = int(s.mem_begin[0])
    s.keep[m0:m0 + 300] = 0
    for at in (None, 0, 299, 128):
        s.keep[m0:m0 + int(s.mem_len[0])] = 0
        if at is not None:
            s.keep[m0 + at] = 1
            s.k[m0 + at], s.v[m0 + at] = 0.5, -2.0
        s.out.fill_(NAN)
        h.cross(s.desc())
        s.check(torch)
        assert (s.out[:s.begin[1]] == (0.0 if at is None else -2.0)).all()


@pytest.mark.parametrize("route", ROUTES)
def test_sharp_scores_and_scales(torch, h, route):
    for sharp, scale, dt in ((30.0, None, "float16"), (1e-3, None, "bfloat16"), (1.0, 0.0, "bfloat16"), (1.0, -0.3, "float16"),
                             (1.0, 4.0, "bfloat16")):
        s = Set(torch, *ROUTES[route], dt=dt, sharp=sharp)
        if scale is not None:
            s.scale = scale
        h.cross(s.desc())
        s.check(torch)


@pytest.mark.parametrize("route", ROUTES)
def test_scores_that_grow_along_the_memory(torch, h, route):
    """Each tile raises the rows' maxima, so every sum is rescaled; and falls, so none is."""
    new, mem, H, Hkv, D = ROUTES[route]
    for sign in (1, -1):
        s = Set(torch, new, mem, H, Hkv, D, gap=0)
        s.q.fill_(1.0)
        ramp = torch.linspace(-3, 3, len(s.k), device="cuda") * sign
        s.k.copy_(ramp.view(-1, 1, 1).expand_as(s.k))
        h.cross(s.desc())
        s.check(torch)


@pytest.mark.parametrize("route", ROUTES)
def test_what_is_not_finite(torch, h, route):
    """A NaN query or state makes its head NaN, a value that is not finite its column; scores of -infinity alone
    give zeros."""
    new, mem, H, Hkv, D = ROUTES[route]
    s = Set(torch, new, mem, H, Hkv, D)
    G = H // Hkv
    s.q[0, 1] = NAN
    m1 = int(s.mem_begin[1])
    s.v[m1 + 130, 0, 5] = INF
    s.v[m1 + 131, Hkv - 1, 6] = NAN
    h.cross(s.desc())
    bad = s.out[:int(s.begin[3])].isnan() | s.out[:int(s.begin[3])].isinf()
    want = torch.zeros_like(bad)
    want[0, 1] = True
    t = slice(int(s.begin[1]), int(s.begin[2]))
    want[t, :G, 5] = True
    want[t, (Hkv - 1) * G:, 6] = True
    assert torch.equal(bad, want)
    s = Set(torch, new, mem, H, Hkv, D)
    s.k[m1 + 131, 0, 3] = NAN
    h.cross(s.desc())
    want = torch.zeros_like(bad)
    want[t, :G] = True
    assert torch.equal(s.out[:int(s.begin[3])].isnan(), want)
    s = Set(torch, new, mem, H, Hkv, D)
    s.q.fill_(1.0)
    m0 = int(s.mem_begin[0])
    s.k[m0:m0 + mem[0]] = -INF
    h.cross(s.desc())
    assert (s.out[:new[0]] == 0).all()


@pytest.mark.parametrize("route", ROUTES)
def test_memories_that_are_shared(torch, h, route):
    """Two requests over one memory, and over parts of it."""
    s = Set(torch, *ROUTES[route])
    s.mem_begin[:], s.mem_len[:] = int(s.mem_begin[1]), 1000
    s.mem_begin[2] += 500
    s.mem_len[2] = 300
    h.cross(s.desc())
    s.check(torch)


@pytest.mark.parametrize("route", ROUTES)
def test_in_place(torch, h, route):
    s = Set(torch, *ROUTES[route])
    want = s.want()
    s.out = s.q
    h.cross(s.desc())
    s.check(torch, want)


def test_no_states_at_all(torch, h):
    for route in ROUTES:
        new, _, H, Hkv, D = ROUTES[route]
        s = Set(torch, new, [0, 0, 0], H, Hkv, D, gap=0)
        assert s.max_mem == 0
        h.cross(s.desc())
        assert (s.out[:sum(new)] == 0).all()
        s.out.fill_(NAN)
        h.cross(s.desc(max_mem=10))
        assert (s.out[:sum(new)] == 0).all()


def test_one_state_gives_its_value(torch, h):
    """To the bit, on every route."""
    for route in ROUTES:
        for dt in ("bfloat16", "float16"):
            new, _, H, Hkv, D = ROUTES[route]
            s = Set(torch, new, [1, 1, 1], H, Hkv, D, dt=dt)
            h.cross(s.desc())
            for b in range(3):
                v = s.v[int(s.mem_begin[b])].repeat_interleave(H // Hkv, dim=0)
                assert torch.equal(s.out[int(s.begin[b]):int(s.begin[b + 1])], v.expand(new[b], H, D))


def test_many_requests(torch, h):
    """More than a block's threads, some without tokens, some without states."""
    new, mem = [i % 3 for i in range(700)], [(i * 37) % 90 for i in range(700)]
    s = Set(torch, new, mem, 2, 1, 32, gap=0)
    h.cross(s.desc())
    s.check(torch)


def test_tokens_repeat_to_the_bit(torch, h):
    for route in ROUTES:
        s = Set(torch, *ROUTES[route], holes=0.1)
        h.cross(s.desc())
        first = s.out.clone()
        for _ in range(10):
            s.out.fill_(NAN)
            h.cross(s.desc())
            assert torch.equal(s.out.view(torch.int16), first.view(torch.int16))


def test_in_graphs_with_other_lengths(torch, h):
    """Captured without a call before it; two graphs of one handle; replays with other lengths and masks."""
    st = torch.cuda.Stream()
    sets = [Set(torch, *ROUTES[r], holes=0.2) for r in ROUTES]
    graphs = []
    torch.cuda.synchronize()
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            h.cross(s.desc(), torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    ends = [int(s.begin[2]) for s in sets]
    for step in range(3):
        for s, g, end in zip(sets, graphs, ends):
            s.mem_len[1] = 1000 - 333 * step
            s.begin[2] = end - step  # the last request takes over tokens of the one before it
            g.replay()
        torch.cuda.synchronize()
        for s in sets:
            s.check(torch)


def test_lengths_that_contradict_the_call(torch):
    for route in ROUTES:
        for name, at, v in (("begin", 3, 10 ** 9), ("begin", 0, -4), ("mem_len", 1, 2 ** 30), ("mem_len", 0, -1), ("mem_begin", 1, -7),
                            ("mem_begin", 0, 2 ** 30)):
            with wt.Handle([]) as h:
                s = Set(torch, *ROUTES[route], pad=5)
                getattr(s, name)[at] = v
                h.cross(s.desc())
                torch.cuda.synchronize()
                assert h.device_status() == wt.WT_EINVAL, (route, name)


def test_states_past_2_gib(torch, h):
    """Offsets of a long memory pass 32 bits."""
    M, Hkv, D = 1 << 19, 20, 128
    k = torch.zeros(M, 2, Hkv, D, dtype=torch.bfloat16, device="cuda")
    k[:, 1] = 1.0
    k[M - 700:].normal_(generator=torch.Generator("cuda").manual_seed(1))
    for new in (1, 80):
        q = torch.randn(new, Hkv, D, device="cuda").bfloat16()
        out = torch.empty_like(q)
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        h.cross(serving.cross_attention(q, out, ints(0, new), k[:, 0], k[:, 1], ints(M - 700), ints(700), max_new=new, max_mem=700))
        want, mag, qk = plain.cross(q, ints(0, new), k[M - 700:, 0], k[M - 700:, 1], ints(0), ints(700), None, D ** -0.5)
        tol = (2.0 ** -8 + 2 * (D / 16 + 4) * 2.0 ** -23 * qk + 2.0 ** -15) * mag + 2.0 ** -8 * want.abs()
        assert ((out.double().cpu() - want).abs() <= tol).all()


def test_more_work_than_a_warp_counts(torch, h):
    """One request of 65536 tokens and 2^20 states: 2^25 cells, of which a few tokens are checked."""
    N, M, H, D = 65536, 1 << 20, 16, 8
    g = torch.Generator("cuda").manual_seed(3)
    q, k, v = (torch.randn(n, H, D, device="cuda", generator=g).bfloat16() for n in (N, M, M))
    out = torch.empty_like(q)
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    h.cross(serving.cross_attention(q, out, ints(0, N), k, v, ints(0), ints(M), max_new=N, max_mem=M))
    some = torch.tensor([0, 1, 255, 256, 30001, N - 1], device="cuda")
    s = torch.einsum("nhd,khd->hnk", q[some].double(), k.double()) * D ** -0.5
    want = torch.einsum("hnk,khd->nhd", torch.softmax(s, dim=2), v.double())
    # the mean of 2^20 values near 0: sum p |v| is below 1, weights are rounded by 2^-8 each, sums in fp32 keep 2^-15
    assert ((out[some].double() - want).abs() <= 2.0 ** -8 + 2.0 ** -15 + 2.0 ** -8 * want.abs()).all()
    assert ((out[some].double() - want).abs().mean() <= 2.0 ** -12)  # the roundings of 2^20 weights cancel


def test_pitches_that_say_nothing(torch, h):
    """Of one state, one kv head, one token: any pitch does."""
    for new in (1, 40):
        s = Set(torch, [new], [1], 4, 1, 64, gap=0)
        d = s.desc()
        d.mem_stride, d.mem_head = 1 << 40, 1 << 40
        if new == 1:
            d.q_stride = 1 << 40
        h.cross(d)
        s.check(torch)


def test_what_is_refused(torch, h):
    def refuse(change, code=wt.WT_EINVAL, holes=None):
        s = Set(torch, [2, 1], [300, 20], 8, 2, 64, holes=holes)
        d = s.desc()
        change(d)
        with pytest.raises(wt.WtError) as e:
            h.cross(d)
        assert e.value.code == code and "wt_cross" in str(e.value), str(e.value)

    def put(**kw):
        return lambda d: [setattr(d, k, v) for k, v in kw.items()]

    refuse(put(dtype=wt.WT_F32), wt.WT_ENOTSUP)
    refuse(put(dtype=9))
    refuse(put(head_dim=136), wt.WT_ENOTSUP)
    for kw in (dict(head_dim=60), dict(heads=7), dict(kv_heads=0), dict(heads=65544), dict(n_req=-1), dict(n_req=65536), dict(n_tokens=-1),
               dict(n_tokens=2 ** 30 + 1), dict(max_new=-1), dict(max_mem=-1), dict(max_mem=2 ** 30 + 1), dict(n_mem=-1), dict(n_mem=2 ** 31),
               dict(scale=float("inf")), dict(q_stride=8), dict(out_stride=516), dict(mem_stride=32), dict(mem_head=68),
               dict(mem_stride=2 ** 41), dict(q=None), dict(out=None), dict(begin=None), dict(k=None), dict(v=None), dict(mem_begin=None),
               dict(mem_len=None), dict(n_tokens=10 ** 7), dict(n_mem=10 ** 7)):
        refuse(put(**kw))
    for name in ("q", "out", "k", "v"):
        refuse(lambda d: setattr(d, name, getattr(d, name) + 8))
    refuse(lambda d: setattr(d, "out", d.k))
    refuse(lambda d: setattr(d, "out", d.q + 16))
    refuse(lambda d: setattr(d, "keep", d.out), holes=0.1)
    assert h.kernel_launches() == 0
    s = Set(torch, [2, 1], [300, 20], 8, 2, 64)
    for kw in (dict(n_tokens=0), dict(n_req=0), dict(max_new=0)):
        d = s.desc()
        put(**kw)(d)
        h.cross(d)
    assert h.kernel_launches() == 0


def test_descriptors_from_tensors(torch):
    s = Set(torch, [2, 1], [300, 20], 8, 2, 64)
    names = dict(q=s.q, out=s.out, begin=s.begin, k=s.k, v=s.v, mem_begin=s.mem_begin, mem_len=s.mem_len)
    for kw in (dict(q=s.q.float()), dict(out=s.out[:1]), dict(k=s.k.half()), dict(v=s.v[:5]), dict(k=s.k[:, :, :32], v=s.v[:, :, :32]),
               dict(v=s.v.transpose(0, 1).contiguous().transpose(0, 1)), dict(begin=s.begin.long()), dict(mem_len=s.mem_len[:1]),
               dict(mem_begin=s.mem_begin.cpu()), dict(q=s.q[:, :, ::2])):
        with pytest.raises(ValueError):
            serving.cross_attention(**{**names, **kw}, max_new=2, max_mem=300)
    with pytest.raises(ValueError):
        s.desc(keep=torch.ones(5, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        s.desc(keep=s.inside)
