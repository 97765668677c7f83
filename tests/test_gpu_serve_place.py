"""wt_place against 64 bits: norms, rotation, axes, pages, and what lies beside them."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve_more as plain

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


FREQ = lambda pairs: [10000.0 ** (-j / max(1, pairs)) for j in range(pairs)]  # noqa: E731


class Set:
    """One call: requests of `new` tokens behind `past` keys each."""

    def __init__(self, torch, new, past, H=4, Hkv=2, D=64, rot=64, page=16, src="f32", dtype="bf16", norm=None, near=False, axes=0,
                 first=0, pad=0, fused=False, seed=0, parts="qkv", eps=1e-6):
        T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
        g = torch.Generator("cuda").manual_seed(seed)
        src, self.dt = T[src], T[dtype]

        def normal(*shape, dtype=torch.float32):
            return torch.randn(shape, device="cuda", generator=g).to(dtype)

        def ints(v):
            return torch.tensor(v, dtype=torch.int32, device="cuda")

        self.begin = ints([sum(new[:b]) for b in range(len(new) + 1)])
        lens = [n + p for n, p in zip(new, past)]
        self.lens, self.max_len, self.page = ints(lens), max(lens + [1]), page
        N = sum(new) + pad
        if fused:
            self.q, self.k, self.v = normal(N, H + 2 * Hkv, D, dtype=src).split((H, Hkv, Hkv), dim=1)
        else:
            self.q, self.k, self.v = normal(N, H, D, dtype=src), normal(N, Hkv, D, dtype=src), normal(N, Hkv, D, dtype=src)
        self.q, self.k, self.v = (t if n in parts else None for n, t in zip("qkv", (self.q, self.k, self.v)))
        nt = T.get(norm)
        self.q_norm, self.k_norm = (None, None) if nt is None else ((1 + 0.2 * normal(D)).to(nt), (1 + 0.2 * normal(D)).to(nt))
        self.eps, self.freq, self.near, self.first = eps, FREQ(rot // 2), near, first
        self.axis = [j % axes for j in range(rot // 2)] if axes else None
        self.pos = (torch.randint(-3000, 3000, (N, axes), device="cuda", generator=g).int() + first) if axes else None
        per = [-(-n // page) for n in lens]
        total = sum(per) + 2
        order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = ints([[order[sum(per[:b]) + j] if j < per[b] else -1 for j in range(max(per + [1]))] for b in range(len(new))])
        self.k_pages, self.v_pages = normal(total, page, Hkv, D, dtype=self.dt), normal(total, page, Hkv, D, dtype=self.dt)
        self.q_out = normal(N, H, D, dtype=self.dt)
        self.before = [t.clone() for t in (self.q_out, self.k_pages, self.v_pages)]

    def desc(self, **kw):
        a = dict(q=self.q, q_out=None if self.q is None else self.q_out, k=self.k, v=self.v, max_len=self.max_len, q_norm=self.q_norm,
                 k_norm=self.k_norm, eps=self.eps, turns=serving.turns(self.freq) if self.freq else None, axis=self.axis,
                 pos=self.pos if self.freq else None, first_pos=self.first, neighbours=self.near)
        a.update(kw)
        return serving.placement(self.begin, self.k_pages, self.v_pages, self.table, self.lens, **a)

    def want(self):
        return plain.place(self.q, self.k, self.v, self.begin, self.lens, self.table, self.page, self.q_norm, self.k_norm, self.eps,
                           self.freq, self.axis, self.pos, self.first, self.near)

    def check(self, torch, want=None):
        """Sums of 8 squares a lane and 5 exchanges, half of their error in the root, its own and two products:
        below 2^-21; the angle (its 32 bits, its conversion, sincospif): below 2^-21 of both elements.  Together
        2^-20 of the pair before the one rounding."""
        qs, rows = self.want() if want is None else want
        u, tiny = torch.finfo(self.dt).eps / 2, 2.0 ** -25 if self.dt == torch.float16 else 2.0 ** -134
        out, kp, vp = (t.double().cpu() for t in (self.q_out, self.k_pages, self.v_pages))

        def near(got, y, mag):
            err = 2.0 ** -20 * mag
            assert ((got - y).abs() <= err + u * (y.abs() + err) + tiny).all(), float(((got - y).abs() / (y.abs() + 1e-9)).max())

        for t, (y, mag) in qs.items():
            near(out[t], y, mag)
        for (p, r), (k, v) in rows.items():
            if k is not None:
                near(kp[p, r], *k)
            if v is not None:
                near(vp[p, r], *v)
        # all else is as it was
        q0, k0, v0 = (t.double().cpu() for t in self.before)
        for t in range(len(out)):
            if t not in qs:
                assert torch.equal(out[t], q0[t])
        keep = torch.ones(kp.shape[:2], dtype=torch.bool)
        for (p, r) in rows:
            keep[p, r] = False
        for got, was, part in ((kp, k0, self.k), (vp, v0, self.v)):
            same = keep if part is not None else torch.ones_like(keep)
            assert torch.equal(got[same], was[same])


CASES = {
    "one token": dict(new=[1], past=[5]),
    "first token": dict(new=[1], past=[0], H=1, Hkv=1, D=8, rot=8, page=1),
    "plain rows": dict(new=[3, 2], past=[4, 0], rot=0),
    "ragged": dict(new=[3, 0, 5, 1], past=[0, 9, 30, 16], page=24, pad=3),
    "gqa 128": dict(new=[9, 4], past=[100, 1], H=8, Hkv=2, D=128, rot=128, page=64, norm="bf16"),
    "neighbours": dict(new=[9, 4], past=[10, 1], D=80, rot=40, near=True, page=24, dtype="f16", norm="f16"),
    "part turned": dict(new=[6], past=[7], D=96, rot=32, dtype="f16", norm="f32"),
    "one pair group": dict(new=[6], past=[7], D=72, rot=8, near=True),
    "widest": dict(new=[2, 3], past=[7, 0], D=256, rot=256, H=3, Hkv=3, norm="f32", page=7),
    "odd width": dict(new=[5], past=[3], D=168, rot=88, H=5, Hkv=1, norm="bf16"),
    "axes": dict(new=[7, 3], past=[0, 4], D=128, rot=128, axes=3, src="bf16", fused=True, norm="bf16"),
    "eight axes": dict(new=[4], past=[0], D=64, rot=64, axes=8, near=True, src="f16", dtype="f16"),
    "far": dict(new=[3], past=[2], D=64, rot=64, first=2 ** 30 - 9),
    "far axes": dict(new=[3], past=[2], D=64, rot=64, axes=2, first=2 ** 31 - 4000),
    "16-bit": dict(new=[3, 1], past=[2, 2], src="f16", dtype="f16", fused=True),
    "keys alone": dict(new=[3, 1], past=[2, 2], parts="k", norm="f32"),
    "values alone": dict(new=[3, 1], past=[2, 2], parts="v"),
    "queries alone": dict(new=[3, 1], past=[2, 2], parts="q", norm="f32"),
    "many requests": dict(new=[1] * 70 + [0] * 5 + [2] * 5, past=[3] * 80, H=2, Hkv=1, D=16, rot=16, page=2),
    "many heads": dict(new=[2], past=[3], H=70, Hkv=35, D=24, rot=24),
    "many tokens": dict(new=[700, 300], past=[0, 11], H=2, Hkv=1, D=32, rot=16, pad=2),
}


@pytest.mark.parametrize("name", CASES)
def test_against_64_bits(torch, h, name):
    s = Set(torch, **CASES[name])
    h.place(s.desc())
    s.check(torch)


def test_thousands_of_requests(torch, h):
    """The search for a token's request over more than 1024 of them, some without tokens."""
    new = [i % 3 for i in range(2500)]
    s = Set(torch, new, [i % 2 for i in range(2500)], H=1, Hkv=1, D=8, rot=8, page=2)
    h.place(s.desc())
    s.check(torch)


def test_in_place(torch, h):
    s = Set(torch, [5, 3], [0, 2], H=4, Hkv=2, D=64, src="bf16", fused=True, norm="bf16")
    want = s.want()
    s.q_out = s.q
    s.before[0] = s.q.clone()
    h.place(s.desc())
    s.check(torch, want)


def test_without_requests(torch, h):
    """Queries of all rows: a rotation by pos, and none at all."""
    s = Set(torch, [6], [0], axes=1, parts="q")
    h.place(serving.placement(q=s.q, q_out=s.q_out, turns=serving.turns(s.freq), pos=s.pos))
    s.check(torch)
    s = Set(torch, [6], [0], rot=0, parts="q", norm="f32")
    h.place(serving.placement(q=s.q, q_out=s.q_out, q_norm=s.q_norm))
    s.check(torch)


@pytest.mark.parametrize("size", [1e30, 1e19, 1e-30, 1e-20, 0.0])
def test_norms_of_large_and_small_numbers(torch, h, size):
    """Squares past fp32's range on either side do not make a norm infinite or zero."""
    s = Set(torch, [3], [0], D=128, rot=64, norm="f32", eps=0.0 if size else 1e-6)
    for t in (s.q, s.k):
        t.mul_(size)
    h.place(s.desc())
    s.check(torch)


def test_what_is_not_finite_stays_in_its_pair(torch, h):
    """Without a norm a NaN reaches its own pair, with one its own head."""
    for norm in (None, "f32"):
        s = Set(torch, [4], [0], norm=norm)
        clean = Set(torch, [4], [0], norm=norm)
        s.q[1, 2, 3] = float("nan")
        h.place(s.desc())
        h.place(clean.desc())
        bad = s.q_out.isnan()
        want = torch.zeros_like(bad)
        if norm:
            want[1, 2] = True
        else:
            want[1, 2, 3] = want[1, 2, 35] = True
        assert torch.equal(bad, want) and torch.equal(s.q_out[~bad], clean.q_out[~bad])
        assert torch.equal(s.k_pages, clean.k_pages) and torch.equal(s.v_pages, clean.v_pages)


def test_attention_finds_what_was_placed(torch, h):
    """Rows go through place and then attend, against attention to the rows themselves in 64 bits."""
    s = Set(torch, [3, 1, 4], [20, 0, 33], H=8, Hkv=2, D=64, norm="bf16")
    h.place(s.desc())
    out = torch.empty_like(s.q_out)
    h.attend(serving.attention(s.q_out, out, s.begin, s.k_pages, s.v_pages, s.table, s.lens, max_new=4, max_len=s.max_len))
    from tests import _serve
    want, mag, qk = _serve.attend(s.q_out, s.begin, None, None, s.k_pages, s.v_pages, s.table, s.lens, 64 ** -0.5)
    tol = (2.0 ** -8 + 2.0 ** -18 * qk + 2.0 ** -15) * mag + 2.0 ** -8 * want.abs()
    assert ((out.double().cpu() - want).abs() <= tol).all()


def test_pages_and_places_that_are_not_there(torch):
    """A page out of range and a place before the first key: the token is not cached, its query is made."""
    for spoil in ("page", "len"):
        with wt.Handle([]) as h:
            s = Set(torch, [3, 2], [14, 0], axes=1)
            qs, rows = s.want()
            if spoil == "page":
                s.table[0, 1] = 10 ** 6
                gone = [(0, 16)]
            else:
                s.lens[1] = 1  # two new tokens: the first has place -1
            want_rows = {}
            old = s.table.clone()
            for b, n, m in ((0, 3, 17), (1, 2, 2)):
                for i in range(n):
                    at = (int(s.lens[b]) - n + i)
                    if at < 0 or not 0 <= int(old[b, at // 16]) < len(s.k_pages):
                        continue
                    t = int(s.begin[b]) + i
                    p = [int(s.pos[t, 0])] * len(s.freq)
                    want_rows[(int(old[b, at // 16]), at % 16)] = (plain.place_head(s.k[t].cpu(), None, 0, s.freq, p, False),
                                                                 plain.place_head(s.v[t].cpu(), None, 0, [], [], False))
            h.place(s.desc())
            torch.cuda.synchronize()
            assert h.device_status() == wt.WT_EINVAL
            s.check(torch, (qs, want_rows))


def test_offsets_that_contradict_the_call(torch):
    """begin past n_tokens and lengths past max_len write nothing outside the buffers."""
    for spoil in ("begin", "len", "negative"):
        with wt.Handle([]) as h:
            s = Set(torch, [3, 2], [4, 0], pad=4)
            if spoil == "begin":
                s.begin[2] = 10 ** 9
            elif spoil == "len":
                s.lens[1] = 2 ** 30
            else:
                s.begin[0] = -5
            h.place(s.desc())
            torch.cuda.synchronize()
            assert h.device_status() == wt.WT_EINVAL


def test_in_a_graph_and_on_a_stream(torch, h):
    """Captured without a call before it, replayed with other inputs and lengths."""
    s = Set(torch, [2, 1], [3, 20], norm="f32")
    d, st = s.desc(), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        h.place(d, torch.cuda.current_stream().cuda_stream)
    for step in range(2):
        s.q.normal_(), s.k.normal_(), s.v.normal_()
        s.lens -= step
        for t, b in zip((s.q_out, s.k_pages, s.v_pages), s.before):
            b.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        s.check(torch)


def test_what_is_refused(torch, h):
    def refuse(change, code=wt.WT_EINVAL, **kw):
        s = Set(torch, [2, 1], [3, 20], **kw)
        d = s.desc()
        change(s, d)
        with pytest.raises(wt.WtError) as e:
            h.place(d)
        assert e.value.code == code and "wt_place" in str(e.value), str(e.value)

    def put(**kw):
        def change(s, d):
            for k, v in kw.items():
                setattr(d, k, v)
        return change

    refuse(put(dtype=wt.WT_F32), wt.WT_ENOTSUP)
    refuse(put(dtype=77))
    refuse(put(in_dtype=wt.WT_F16), wt.WT_ENOTSUP)
    refuse(put(norm_dtype=wt.WT_I8), wt.WT_ENOTSUP, norm="f32")
    refuse(put(head_dim=264), wt.WT_ENOTSUP)
    for kw in (dict(head_dim=60), dict(rot_dim=12), dict(rot_dim=72), dict(rot_dim=-8), dict(flags=6), dict(heads=0), dict(kv_heads=0),
               dict(n_tokens=-1), dict(n_tokens=2 ** 30 + 1), dict(n_req=-1), dict(first_pos=-1), dict(max_len=-1), dict(page=0),
               dict(table_stride=1), dict(q_stride=8), dict(out_stride=4 * 64 + 4), dict(k_stride=2 ** 41), dict(begin=None),
               dict(len=None), dict(turns=None), dict(q_out=None), dict(k_pages=None), dict(table=None), dict(n_tokens=10 ** 6)):
        refuse(put(**kw))
    refuse(put(eps=-1.0), norm="f32")
    refuse(put(eps=float("nan")), norm="f32")
    refuse(put(axes=9), axes=2)
    refuse(put(pos_stride=1), axes=2)
    refuse(lambda s, d: d.axis.__setitem__(5, 2), axes=2)
    for name in ("q", "k", "v", "q_out", "k_pages", "v_pages"):
        refuse(lambda s, d: setattr(d, name, getattr(d, name) + 8))
    refuse(lambda s, d: setattr(d, "q_out", d.k_pages))
    refuse(lambda s, d: setattr(d, "v_pages", d.k_pages))
    refuse(lambda s, d: setattr(d, "q_out", d.q))  # of another type
    refuse(lambda s, d: setattr(d, "k_pages", d.k), src="bf16")
    # q_out over k, which is q: only q itself may be written in place
    refuse(lambda s, d: (setattr(d, "q_out", d.q), setattr(d, "k", d.q), setattr(d, "k_stride", d.q_stride)), src="bf16")
    assert h.kernel_launches() == 0


def test_nothing_to_do(torch, h):
    s = Set(torch, [2], [3])
    for kw in (dict(n_tokens=0), dict(n_req=0), dict(q=None, k=None, v=None)):
        d = s.desc()
        for k, v in kw.items():
            setattr(d, k, v)
        h.place(d)
    assert h.kernel_launches() == 0
    s = Set(torch, [0, 0], [3, 2], pad=5)  # rows that no request holds
    h.place(s.desc())
    s.check(torch)


def test_descriptors_from_tensors(torch):
    s = Set(torch, [2, 1], [3, 20], axes=2, norm="f32")
    bad = [dict(q=s.q.double()), dict(q=s.q[:, :, ::2]), dict(q_out=s.q_out[:2]), dict(q_out=None), dict(k=s.k[:2]), dict(v=s.v[:, :1]),
           dict(q_norm=s.q_norm[:8]), dict(k_norm=s.k_norm.half()), dict(turns=serving.turns(s.freq)[:3]), dict(turns=s.lens),
           dict(axis=[2] * 32), dict(axis=[0] * 3), dict(pos=s.pos.long()), dict(pos=None), dict(max_len=0), dict(max_len=10 ** 6),
           dict(q=s.q.cpu())]
    for kw in bad:
        with pytest.raises(ValueError):
            s.desc(**kw)
    with pytest.raises(ValueError):
        serving.placement(q=s.q, q_out=s.q_out, turns=serving.turns(s.freq))  # no place
    with pytest.raises(ValueError):
        serving.placement(k=s.k, k_pages=s.k_pages)
    with pytest.raises(ValueError):
        serving.placement()
