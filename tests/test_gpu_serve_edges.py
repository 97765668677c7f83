"""Placing and attention to memories at the edges of what a call may hold: parts without the rest, the most rows, long sums,
offsets that lie, and what stands around the outputs."""
import math

import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve_more as plain
from tests.test_gpu_serve_cross import ROUTES
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


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_sums_of_2_20_states(torch, h, dt):
    """One request of 65536 tokens and 2^20 states, 2^25 cells: tokens at the borders of row tiles that two CTAs share,
    each by itself, of values near 1 as well as near 0."""
    N, M, H, D = 65536, 1 << 20, 16, 8
    dt = getattr(torch, dt)
    u = torch.finfo(dt).eps / 2
    g = torch.Generator("cuda").manual_seed(5)
    q, k, v = (torch.randn(n, H, D, device="cuda", generator=g).to(dt) for n in (N, M, M))
    v[:, :, 0] = 1.0
    v[:, :, 1] = 1.0 + 0.25 * v[:, :, 1]
    out = torch.full_like(q, float("nan"))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    h.cross(serving.cross_attention(q, out, ints(0, N), k, v, ints(0), ints(M), max_new=N, max_mem=M))
    torch.cuda.synchronize()
    assert not out.isnan().any()
    # row tiles of 256 tokens and 8192 key tiles, 256 to a head; a CTA to an SM
    tiles, sms = (N // 256) * (M // 128), torch.cuda.get_device_properties(0).multi_processor_count
    per = -(-H * tiles // sms)
    cut = {per * c % tiles // (M // 128) for c in (1, sms // 4, sms // 2, sms - 1)}
    some = sorted({t for r in cut | {0, N // 256 - 1} for t in (256 * r, 256 * r + 127, 256 * r + 128, 256 * r + 255)})
    some = torch.tensor(some, device="cuda")
    p = torch.softmax(torch.einsum("nhd,khd->hnk", q[some].double(), k.double()) * D ** -0.5, dim=2)
    want = torch.einsum("hnk,khd->nhd", p, v.double())
    # A weight's rounding is up to u of it, and 2^20 of them cancel: their part of a sum p v has a standard deviation of
    # u sqrt(sum p^2 v^2 / 3), below u 2^-8 for the sharpest rows here (|q|^2 = 28); eight of them.  The sums: as kept
    # in wt_serve.h, a tenth of u, and 2^-17 for what is added up to nearest.
    off = out[some].double() - want
    sizes = torch.einsum("hnk,khd->nhd", p, v.double().abs())
    assert (off.abs() <= u * want.abs() + 8 * u * 2.0 ** -8 + (0.1 * u + 2.0 ** -17) * sizes).all()
    assert off[:, :, :2].mean().abs() <= 0.2 * u  # near 1: the outputs' roundings go both ways, or are none
    assert (off[:, :, 2:].abs().mean(dim=(1, 2)) <= 2.0 ** -12).all()  # of each token, by values of both signs: zeros are off by 2^-10


LONG = {  # new, requests, heads, kv heads, D: one memory for all, so that CTAs have long runs of it
    "8 rows, heads together": (1, 310, 4, 4, 64), "8 rows": (2, 330, 3, 1, 128), "16 rows": (4, 320, 12, 4, 72), "32 rows": (8, 310, 16, 4, 64),
    "32 rows of 40": (8, 310, 8, 2, 40), "one row tile": (32, 160, 4, 1, 64), "one row tile of 128": (32, 160, 4, 1, 128),
    "two row tiles": (64, 160, 4, 1, 56), "two row tiles of 128": (70, 160, 4, 1, 120)}


@pytest.mark.parametrize("name", LONG)
@pytest.mark.parametrize("dt,M", [("float16", 40001), ("bfloat16", 300007)])
@pytest.mark.parametrize("holes", [False, True])
def test_long_memories_on_every_route(torch, h, name, dt, M, holes):
    """Values near 1 over more states than one sum takes, and late a state that outweighs all before it by half, so that what was
    summed up has to follow a new reference."""
    new, B, H, Hkv, D = LONG[name]
    dt = getattr(torch, dt)
    u = torch.finfo(dt).eps / 2
    g = torch.Generator("cuda").manual_seed(7)
    k, v = (torch.randn(M, Hkv, D, device="cuda", generator=g).to(dt) for _ in range(2))
    q = torch.randn(new * B, H, D, device="cuda", generator=g).to(dt)
    q[:, :, 0], k[:, :, 0] = 1.0, 0.0
    v = (torch.linspace(1, 1.9, D, device="cuda") + 0.25 * v.float()).to(dt)
    k[M * 3 // 4, :, 0] = D ** 0.5 * math.log(M)
    v[M * 3 // 4] += 1.0
    keep = None
    if holes:
        keep = (torch.rand(M, device="cuda", generator=g) < 0.9).to(torch.uint8)
        keep[M * 3 // 4] = 1
        k[keep == 0], v[keep == 0] = float("nan"), float("inf")
    out = torch.full_like(q, float("nan"))
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    h.cross(serving.cross_attention(q, out, ints([new * b for b in range(B + 1)]), k, v, ints([0] * B), ints([M] * B), max_new=new,
                                    max_mem=M, keep=keep))
    torch.cuda.synchronize()
    assert not out.isnan().any()
    some = torch.arange(0, new * B, new * B // 40 | 1, device="cuda")
    rows = slice(None) if keep is None else keep != 0
    off, near = [], []
    for x in range(H):
        ks, vs = k[rows, x * Hkv // H].double(), v[rows, x * Hkv // H].double()
        p = torch.softmax(q[some, x].double() @ ks.t() * D ** -0.5, dim=1)
        want, sizes = p @ vs, p @ vs.abs()
        off.append((out[some, x].double() - want) / want)
        # the late state's weight and the output are rounded by u each, the others' roundings cancel (eight deviations of
        # u sqrt(sum p^2 v^2 / 3)), scores are off by 2 (D / 16 + 4) 2^-23 of sums |q k|, here up to 12 + log M, and sums as above
        late = p.amax(dim=1, keepdim=True)
        rest = (p ** 2 @ vs ** 2 - (late * vs[p.argmax(dim=1)]) ** 2).clamp(min=0).sqrt()
        near.append((2 * u * want + u * late * 3 + 8 * u * rest + (2 * (D / 16 + 4) * 2.0 ** -23 * 40 + 0.1 * u + 2.0 ** -17) * sizes) / want)
    off, near = torch.stack(off), torch.stack(near)
    assert (off.abs() <= near).all(), float((off.abs() / near).max())
    assert off.mean().abs() <= 0.25 * u, float(off.mean() / u)


@pytest.mark.parametrize("D,kv", [(64, 1), (64, 2), (128, 1)])
@pytest.mark.parametrize("more", [1, 15, 33, 70])
def test_memories_a_little_longer_than_one_sum_takes(torch, h, D, kv, more):
    """Of the last cell only some warps have states; the others have set nothing aside, whatever an earlier call left there."""
    B, dt = 400, torch.float16
    cell = 4 // kv * (32 if D <= 64 else 16)  # states that the warps of a head take at once
    M = 8192 * cell // (32 if D <= 64 else 16)
    g = torch.Generator("cuda").manual_seed(9)
    k, v = (torch.randn(M + 9000, kv, D, device="cuda", generator=g).to(dt) for _ in range(2))
    v += 100.0
    q = torch.randn(B, kv, D, device="cuda", generator=g).to(dt)
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for n in (M + 9000, M + more):
        out = torch.full_like(q, float("nan"))
        h.cross(serving.cross_attention(q, out, ints(*range(B + 1)), k, v, ints(*[0] * B), ints(*[n] * B), max_new=1, max_mem=n))
        torch.cuda.synchronize()
        for x in range(kv):
            p = torch.softmax(q[:, x].double() @ k[:n, x].double().t() * D ** -0.5, dim=1)
            want = p @ v[:n, x].double()
            # the output's rounding, an eighth of it for the weights', and a fifth for the sums
            assert ((out[:, x].double() - want).abs() <= (1 + 0.125 + 0.2) * 2.0 ** -11 * want.abs()).all(), (n, x)


def guarded(torch, t, rows):
    """A copy of t between `rows` rows of other numbers, and the whole buffer."""
    g = torch.Generator("cuda").manual_seed(11)
    whole = torch.randn((len(t) + 2 * rows,) + t.shape[1:], device="cuda", generator=g).to(t.dtype)
    whole[rows:rows + len(t)] = t
    return whole[rows:rows + len(t)], whole


def bits(torch, t):
    return t.contiguous().view(torch.int16).clone()


@pytest.mark.parametrize("spoil", ["begin", "len", "negative"])
def test_placing_by_offsets_that_lie_writes_its_own_rows(torch, spoil):
    """The rows of the request that lies are those of its clamped numbers; all others, and what stands beside the
    buffers, are as they should be."""
    with wt.Handle([]) as h:
        s = Place(torch, [3, 2], [4, 0], pad=4)
        wholes = []
        for name in ("q_out", "k_pages", "v_pages"):
            t, whole = guarded(torch, getattr(s, name), 3)
            setattr(s, name, t)
            wholes.append(whole)
        s.before = [t.clone() for t in (s.q_out, s.k_pages, s.v_pages)]
        around = [torch.cat([bits(torch, w[:3]), bits(torch, w[-3:])]) for w in wholes]
        if spoil == "begin":  # up to the last row, of which the last two have places
            s.begin[2] = len(s.q)
            want = s.want()
            s.begin[2] = 10 ** 9
        elif spoil == "len":  # up to max_len
            s.lens[1] = s.max_len
            want = s.want()
            s.lens[1] = 2 ** 30
        else:
            want = s.want()
            s.begin[0] = -5
        h.place(s.desc())
        torch.cuda.synchronize()
        assert h.device_status() == wt.WT_EINVAL
        s.check(torch, want)
        for w, was in zip(wholes, around):
            assert torch.equal(torch.cat([bits(torch, w[:3]), bits(torch, w[-3:])]), was)


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("name,at,v", [("begin", 3, 10 ** 9), ("begin", 0, -4), ("mem_len", 1, 2 ** 30), ("mem_len", 0, -1), ("mem_begin", 1, -7),
                                       ("mem_begin", 0, 2 ** 30)])
def test_attending_by_lengths_that_lie_writes_its_own_rows(torch, route, name, at, v):
    """As above: the other requests' results are right, and rows that the clamped numbers do not hold are as they were."""
    with wt.Handle([]) as h:
        s = Cross(torch, *ROUTES[route], pad=5)
        N, M = len(s.q), len(s.k)
        s.out, whole = guarded(torch, s.out, 300)
        t = getattr(s, name)
        t[at] = v
        # the clamped numbers
        begin, mem, lens = s.begin.tolist(), s.mem_begin.tolist(), s.mem_len.tolist()
        begin[0], begin[3] = max(begin[0], 0), min(begin[3], N, begin[2] + s.max_new)
        for b in range(3):
            mem[b] = min(max(mem[b], 0), M)
            lens[b] = min(max(lens[b], 0), s.max_mem, M - mem[b])
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        want = plain.cross(s.q, ints(begin), s.k, s.v, ints(mem), ints(lens), None, s.scale)
        before = bits(torch, whole)
        h.cross(s.desc())
        torch.cuda.synchronize()
        assert h.device_status() == wt.WT_EINVAL
        s.check(torch, want)  # of a request that the gaps' NaN reach nothing is asked
        for b in range(3):
            if not (name.startswith("mem") and b == at):
                assert not want[0][begin[b]:begin[b + 1]].isnan().any()
        after = bits(torch, whole)
        held = torch.zeros(len(whole), dtype=torch.bool, device="cuda")
        held[300 + begin[0]:300 + begin[3]] = True
        assert torch.equal(after[~held], before[~held])
