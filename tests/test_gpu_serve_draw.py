"""Handle.probs against 64-bit softmax, and Handle.verify against exact integer arithmetic.

Tolerance of a probability: expf is off by 2 ulp, its argument (l - m) / t by two roundings of its
value, the sum by at most 2^-20 (32 terms in a chain, then trees), and three more roundings; below
2^-126 a subnormal's spacing."""
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


def close(torch, p, l, temp):
    p, l = p.double().cpu(), l.double().cpu()
    for r in range(l.shape[0]):
        t = 1.0 if temp is None else float(temp[r])
        m = l[r].max()
        if m == -_serve.INF:
            assert (p[r] == 0).all()
        elif t > 0:
            x = (l[r] - m) / t
            want = torch.softmax(x, dim=0)
            tol = want * (2.0 ** -20 + 2.0 ** -22 * x.abs().clamp(max=200)) + 2.0 ** -140
            assert ((p[r] - want).abs() <= tol).all(), (r, float(((p[r] - want).abs() / tol).max()))
        else:
            want = torch.zeros_like(l[r])
            want[int((l[r] == m).nonzero()[0])] = 1
            assert torch.equal(p[r], want)


@pytest.mark.parametrize("rows,V", [(1, 1), (2, 2), (3, 31), (1, 257), (5, 1000), (2, 4099), (160, 4099), (1, 32000), (3, 50021),
                                    (2, 128256), (1, 131073), (2, 262144), (1, 600011), (400, 97)])
def test_probabilities(torch, h, rows, V):
    g = torch.Generator("cuda").manual_seed(rows * V)
    l = torch.randn(rows, V, device="cuda", generator=g) * 4
    temp = torch.tensor([(0.0, 1.0, 0.25, 3.0, -1.0)[i % 5] for i in range(rows)], device="cuda")
    for t in (None, temp):
        p = torch.full((rows, V), _serve.NAN, device="cuda")
        h.probs(serving.probabilities(l, p, temperature=t))
        torch.cuda.synchronize()
        close(torch, p, l, t)


def test_masked_rows_ties_and_extremes(torch, h):
    low, big = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    l = torch.randn(12, 5003, device="cuda")
    l[0] = -_serve.INF                      # nothing left
    l[1], l[1, 4000] = -_serve.INF, -3.0    # one token left
    l[2] = low                              # all masked with the type's lowest value: equal shares
    l[3, ::2] = low
    l[4] = 7.0                              # ties
    l[5, 100:] = big
    l[6, 3], l[6, 4] = big, low
    l[7, :4999] = -_serve.INF
    l[8] = 0.0
    l[9] *= 1000
    for temp in (None, torch.zeros(12, device="cuda"), torch.full((12,), 0.1, device="cuda"), torch.full((12,), 1e-30, device="cuda"),
                 torch.full((12,), 1e30, device="cuda")):
        p = torch.full_like(l, _serve.NAN)
        h.probs(serving.probabilities(l, p, temperature=temp))
        torch.cuda.synchronize()
        close(torch, p, l, temp)


def test_nan_and_infinity(torch, h):
    l = torch.randn(4, 70000, device="cuda")
    l[0, 69999], l[1, 5], l[2, 40000] = _serve.NAN, _serve.INF, _serve.NAN
    temp = torch.tensor([1.0, 0.5, 0.0, 1.0], device="cuda")
    p = torch.zeros_like(l)
    h.probs(serving.probabilities(l, p, temperature=temp))
    torch.cuda.synchronize()
    assert torch.isnan(p[0]).all() and torch.isnan(p[1]).all() and p[2].sum() == 1
    close(torch, p[3:], l[3:], None)


def test_strides_in_place_and_graph(torch, h):
    flat = torch.randn(9 * 1010 + 1, device="cuda")
    l = torch.as_strided(flat, (9, 1003), (1010, 1), 1)
    want, keep = l.clone(), flat.clone()
    out = torch.full((9, 1100), _serve.NAN, device="cuda")
    h.probs(serving.probabilities(l, out[:, 5:1008]))
    torch.cuda.synchronize()
    close(torch, out[:, 5:1008], want, None)
    assert torch.isnan(out[:, :5]).all() and torch.isnan(out[:, 1008:]).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h.probs(serving.probabilities(l, l), s.cuda_stream)
    s.synchronize()
    close(torch, l, want, None)
    hole = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(hole, (9, 1003), (1010, 1), 1).fill_(False)
    assert torch.equal(flat[hole], keep[hole])
    g = torch.cuda.CUDAGraph()
    d = serving.probabilities(want, out[:, 5:1008])
    with torch.cuda.graph(g):
        h.probs(d, torch.cuda.current_stream().cuda_stream)
    want.mul_(-1)
    g.replay()
    torch.cuda.synchronize()
    close(torch, out[:, 5:1008], want, None)


def test_probs_refusals(torch, h):
    l, p = torch.randn(3, 50, device="cuda"), torch.empty(3, 50, device="cuda")

    def refused(**change):
        d = serving.probabilities(l, p)
        for k, v in change.items():
            setattr(d, k, v)
        with pytest.raises(wt.WtError) as e:
            h.probs(d)
        assert e.value.code == wt.WT_EINVAL and "wt_probs" in str(e.value)

    refused(logits=None), refused(p=None), refused(rows=-1), refused(vocab=-1), refused(ldl=49), refused(ldp=49)
    refused(p=l.data_ptr() + 4), refused(p=l.data_ptr(), ldp=51), refused(rows=1 << 27), refused(logits=l.data_ptr() + 2)
    with pytest.raises(ValueError):
        serving.probabilities(l.half(), p)
    with pytest.raises(ValueError):
        serving.probabilities(l, p, temperature=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        serving.probabilities(l.t(), p.t())
    h.probs(serving.probabilities(l[:0], p[:0]))
    h.probs(serving.probabilities(l[:, :0], p[:, :0]))


# ------------------------------------------------------------------ verification

def drafts(torch, counts, V, sharp, certain, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    B, n = len(counts), sum(counts)
    begin = torch.tensor([sum(counts[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    row = torch.tensor([sum(counts[:b]) + b + i for b in range(B) for i in range(counts[b])], device="cuda").long()
    l = torch.randn(n + B, V, device="cuda", generator=g) * sharp
    p = torch.softmax(l, dim=1)
    q = None if certain else torch.softmax(l[row] + torch.randn(n, V, device="cuda", generator=g), dim=1)
    d = (l[row].argmax(dim=1) if n else torch.zeros(0, device="cuda")).int()
    u, w = torch.rand(n, device="cuda", generator=g), torch.rand(B, device="cuda", generator=g)
    return p, q, d, begin, u, w


def run(torch, h, p, q, d, begin, u, w, most, stream=0):
    B = len(begin) - 1
    acc = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    tok = torch.full((B, most + 1), -7, dtype=torch.int32, device="cuda")
    h.verify(serving.verification(p, d, begin, u, w, acc, tok, q=q), stream)
    torch.cuda.synchronize()
    return acc.tolist(), tok.tolist()


@pytest.mark.parametrize("V", [1, 2, 33, 4097, 8200, 50021, 128256])
@pytest.mark.parametrize("counts", [[0], [1], [3], [0, 2, 5, 0], [4] * 9, [40, 33]])
@pytest.mark.parametrize("certain", [False, True])
def test_verification_is_exact(torch, h, V, counts, certain):
    for seed, sharp in ((1, 0.5), (2, 6.0)):
        a = drafts(torch, counts, V, sharp, certain, seed)
        most = max(counts) + 1
        assert run(torch, h, *a, most) == _serve.verify(*a, most)


def test_random_numbers_at_their_ends(torch, h):
    p, q, d, begin, u, w = drafts(torch, [2, 2, 2], 9000, 1.0, False)
    eps = 2.0 ** -24
    for lo in (0.0, eps, 0.5, 1 - eps):
        for hi in (0.0, eps, 0.5, 1 - eps):
            u.fill_(lo), w.fill_(hi)
            assert run(torch, h, p, q, d, begin, u, w, 2) == _serve.verify(p, q, d, begin, u, w, 2)


def test_rows_that_leave_nothing(torch, h):
    p, q, d, begin, u, w = drafts(torch, [1, 1, 1, 1, 0], 3001, 1.0, False)
    u.fill_(1 - 2.0 ** -24)
    p[0], q[0] = 0.0, 1.0 / 3001                              # refused, p empty: -1
    q[1] = p[2]                                               # p == q; u q < p stays
    p[4, int(d[2])], q[2] = 0.0, torch.clamp(p[4] * 2, min=1e-6)  # refused, nothing left of p - q: from p
    p[6] = torch.where(torch.arange(3001, device="cuda") == 77, 1.0, 0.0)
    p[8] = 0.0
    got = run(torch, h, p, q, d, begin, u, w, 1)
    assert got == _serve.verify(p, q, d, begin, u, w, 1)
    assert got[1][0] == [-1, -1] and got[1][4][0] == -1 and got[1][2][0] >= 0
    p[0], p[4] = _serve.NAN, -1.0
    assert run(torch, h, p, q, d, begin, u, w, 1) == _serve.verify(p, q, d, begin, u, w, 1)
    p.fill_(3.0)  # weights above 1 count as 1
    assert run(torch, h, p, q, d, begin, u, w, 1) == _serve.verify(p, q, d, begin, u, w, 1)


def test_the_draw_follows_the_probabilities(torch, h):
    """Over all u_draw on a grid, each token is drawn in proportion to what is left of it."""
    V, n = 8, 4096
    p = torch.tensor([0.4, 0.1, 0.0, 0.05, 0.2, 0.05, 0.15, 0.05], device="cuda").expand(2, V)
    q = torch.tensor([[0.2, 0.3, 0.1, 0.0, 0.1, 0.1, 0.1, 0.1]], device="cuda")
    left = torch.clamp(p[0] - q[0], min=0)
    want = (left / left.sum()).tolist()
    P, Q = p.repeat(n, 1), q.repeat(n, 1)
    begin = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    d = torch.full((n,), 2, dtype=torch.int32, device="cuda")  # p is 0 there: refused
    w = (torch.arange(n, device="cuda") + 0.5) / n
    acc, tok = run(torch, h, P, Q, d, begin, torch.rand(n, device="cuda"), w, 1)
    assert set(acc) == {0}
    got = torch.bincount(torch.tensor([t[0] for t in tok]), minlength=V).double() / n
    assert max(abs(float(a) - b) for a, b in zip(got, want)) <= 1.0 / n + 1e-6


def test_strides_streams_and_graph(torch, h):
    p, q, d, begin, u, w = drafts(torch, [3, 0, 2], 5003, 2.0, False)
    P = torch.full((8, 5100), _serve.NAN, device="cuda")
    Q = torch.full((5, 5011), _serve.NAN, device="cuda")
    P[:, 3:5006], Q[:, 1:5004] = p, q
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want = _serve.verify(p, q, d, begin, u, w, 3)
    assert run(torch, h, P[:, 3:5006], Q[:, 1:5004], d, begin, u, w, 3, s.cuda_stream) == want
    acc, tok = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    desc = serving.verification(p, d, begin, u, w, acc, tok, q=q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.verify(desc, torch.cuda.current_stream().cuda_stream)
    u.copy_(u.flip(0).clone()), w.copy_(w.flip(0).clone())
    g.replay()
    torch.cuda.synchronize()
    assert (acc.tolist(), tok.tolist()) == _serve.verify(p, q, d, begin, u, w, 3)


def test_values_outside_the_descriptor(torch):
    p, q, d, begin, u, w = drafts(torch, [2, 2], 300, 1.0, False)
    d[0], d[3] = 300, -4
    with wt.Handle([]) as h:
        assert run(torch, h, p, q, d, begin, u, w, 2) == _serve.verify(p, q, d, begin, u, w, 2)
        assert h.device_status() == wt.WT_EINVAL
    p, q, d, begin, u, w = drafts(torch, [2, 2], 300, 1.0, False)
    for bad in ([0, 9, 4], [-3, 2, 4], [2, 0, 4], [0, 2, 1 << 30]):
        with wt.Handle([]) as h:
            acc, tok = run(torch, h, p, q, d, torch.tensor(bad, dtype=torch.int32, device="cuda"), u, w, 2)
            assert h.device_status() == wt.WT_EINVAL
            assert all(0 <= a <= 2 for a in acc) and all(-1 <= t < 300 for r in tok for t in r)


def test_verify_refusals(torch, h):
    a = drafts(torch, [2, 1], 50, 1.0, False)
    p, q, d, begin, u, w = a
    acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")

    def refused(**change):
        desc = serving.verification(p, d, begin, u, w, acc, tok, q=q)
        for k, v in change.items():
            setattr(desc, k, v)
        with pytest.raises(wt.WtError) as e:
            h.verify(desc)
        assert e.value.code == wt.WT_EINVAL and "wt_verify" in str(e.value)

    for name in ("p", "drafted", "begin", "u", "u_draw", "accepted", "tokens"):
        refused(**{name: None})
    refused(vocab=0), refused(vocab=(1 << 18) + 1), refused(n_req=-1), refused(n_drafted=-1), refused(max_draft=-1)
    refused(ldp=49), refused(ldq=49), refused(n_drafted=1 << 28), refused(tokens=tok.data_ptr() + 1)
    for bad in (dict(p=p[:-1]), dict(q=q[:, :-1]), dict(u=u[:-1]), dict(drafted=d.long()), dict(tokens=tok.t()), dict(p=p.double())):
        args = dict(p=p, drafted=d, begin=begin, u=u, u_draw=w, accepted=acc, tokens=tok, q=q)
        args.update(bad)
        with pytest.raises(ValueError):
            serving.verification(**args)


def test_offsets_past_32_bits(torch, h):
    far = torch.empty((1 << 31) + 5000, device="cuda")
    l = far.as_strided((3, 4999), (1 << 30, 1))
    l.copy_(torch.randn(3, 4999, device="cuda"))
    near = l.contiguous()
    h.probs(serving.probabilities(l, l))
    torch.cuda.synchronize()
    close(torch, l, near, None)
    p, q, d, begin, u, w = drafts(torch, [2], 4999, 2.0, False)
    l.copy_(p)
    assert run(torch, h, l, q, d, begin, u, w, 2) == _serve.verify(p, q, d, begin, u, w, 2)
