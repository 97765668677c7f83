"""wt_logprobs against 64 bits: log probabilities, entropy, the likeliest tokens, and rows that are not ordinary."""
import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve_more as plain

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


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
    def __init__(self, torch, rows, V, given=1, top=5, temp=True, std=3.0, seed=0, pitch=0, shift=0):
        g = torch.Generator("cuda").manual_seed(seed)
        flat = torch.randn(rows * (V + pitch) + shift, device="cuda", generator=g) * std
        self.logits = flat[shift:].view(rows, V + pitch)[:, :V]
        self.temp = 0.3 + torch.rand(rows, device="cuda", generator=g) if temp else None
        self.given = torch.randint(0, V, (rows, given), device="cuda", generator=g).int() if given else None
        self.given_lp = torch.full((rows, given), 77.0, device="cuda") if given else None
        self.entropy = torch.full((rows,), 77.0, device="cuda")
        self.top = torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None
        self.top_lp = torch.full((rows, top), 77.0, device="cuda") if top else None

    def desc(self, **kw):
        a = dict(given=self.given, given_lp=self.given_lp, entropy=self.entropy, top=self.top, top_lp=self.top_lp, temperature=self.temp)
        a.update(kw)
        return serving.log_probabilities(self.logits, **a)

    def check(self, torch, rows=None):
        """x = (l - m) k: the difference, the factor and the product each rounded, 3 x 2^-24 of x; 2^x within 2^-22;
        a thread adds V / 256 numbers at most, 16 at once.  Weighted by p: log S is off by
        2^-21 (1 + mean |x|) + V 2^-36; log p by that and 2^-22 |x|; the entropy's second sum also by 2^-21 mean x^2."""
        V = self.logits.shape[1]
        for r in range(len(self.logits)) if rows is None else rows:
            t = 1.0 if self.temp is None else float(self.temp[r])
            l = self.logits[r].cpu()
            lp, H, m1, m2 = plain.logprobs(l, t)
            tol = 2.0 ** -21 * (1 + m1) + V * 2.0 ** -36
            assert abs(float(self.entropy[r]) - H) <= tol + 2.0 ** -21 * (m1 + m2), (r, float(self.entropy[r]), H)

            def near(got, want):
                got = got.double().cpu()
                assert torch.equal(got == -INF, want == -INF)
                some = want > -INF
                assert ((got - want)[some].abs() <= (tol + 2.0 ** -21 * want.abs())[some]).all(), (got, want)

            if self.given is not None:
                v = self.given[r].cpu().long()
                near(self.given_lp[r], torch.where(v >= 0, lp[v.clamp(min=0)], torch.zeros(len(v), dtype=torch.float64)))
            if self.top is not None:
                want = plain.top(l, self.top.shape[1])
                assert self.top[r].tolist() == want, r
                near(self.top_lp[r], torch.tensor([-INF if v < 0 else float(lp[v]) for v in want], dtype=torch.float64))


@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (2, 31), (5, 257), (2, 4097), (3, 8191), (1, 32000), (700, 1000), (7, 50021), (2, 128256),
                                    (1, 300001)])
@pytest.mark.parametrize("given,top", [(1, 5), (0, 32), (4, 0)])
def test_against_64_bits(torch, h, rows, V, given, top):
    s = Set(torch, rows, V, given, top, temp=V % 2 == 1, seed=V)
    h.logprobs(s.desc())
    s.check(torch, rows=range(0, rows, max(1, rows // 12)))


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_rows_at_any_alignment(torch, h, shift):
    s = Set(torch, 5, 5003, 2, 7, pitch=shift, shift=4 - shift)
    h.logprobs(s.desc())
    s.check(torch)


@pytest.mark.parametrize("n_top", [1, 2, 31, 32])
def test_equal_logits_in_the_order_of_their_tokens(torch, h, n_top):
    s = Set(torch, 4, 20011, 1, n_top)
    s.logits.copy_(s.logits.round())  # many ties
    s.logits[1] = 2.5
    s.logits[2, ::2], s.logits[2, 1::2] = 0.0, -0.0
    s.logits[3].fill_(-INF)
    s.logits[3, 15000:15010] = 1.0
    s.given[:, 0] = 15003
    h.logprobs(s.desc())
    s.check(torch)


def test_ascending_and_descending_rows(torch, h):
    """Every logit a new largest one, and none after the first."""
    s = Set(torch, 2, 40000, 2, 32)
    s.logits.copy_(torch.linspace(-5, 5, 40000, device="cuda").expand(2, -1))
    s.logits[1] = s.logits[1].flip(0).clone()
    h.logprobs(s.desc())
    s.check(torch)


@pytest.mark.parametrize("step", [5.0, 30.0, 80.0, 300.0])
def test_rows_that_rise_late(torch, h, step):
    """The first thousands of logits far below the others, which their sums were against."""
    s = Set(torch, 4, 30000, 2, 20, temp=False)
    s.logits[0, 9000:] += step
    s.logits[1, 29990:] += step
    s.logits[2, 5000:] += step
    s.logits[2, 15000:] += step
    s.logits[3] += torch.arange(30000, device="cuda") // 4096 * step
    h.logprobs(s.desc())
    s.check(torch)


def test_masked_rows(torch, h):
    """Fewer tokens left than are asked for, one, and none; a given token that is masked."""
    s = Set(torch, 4, 9000, 2, 6)
    for r, n in enumerate((4, 1, 0, 6000)):
        gone = torch.randperm(9000, generator=torch.Generator().manual_seed(r))[n:].cuda()
        s.logits[r, gone] = -INF
        s.given[r, 0] = int(gone[0])
    h.logprobs(s.desc())
    s.check(torch)
    assert s.top[2].tolist() == [-1] * 6 and s.given_lp[2].tolist() == [-INF] * 2 and float(s.entropy[2]) == 0.0


def test_lowest_numbers_as_masks(torch, h):
    """A mask of fp32's lowest number leaves tokens that count, of weight 0; a row of it alone is uniform."""
    low = torch.finfo(torch.float32).min
    s = Set(torch, 2, 5000, 1, 8)
    s.logits[0, 5:] = low
    s.logits[1] = low
    h.logprobs(s.desc())
    assert s.top[1].tolist() == list(range(8)) and s.top[0].tolist()[5:] == [5, 6, 7]
    import math
    assert abs(float(s.entropy[1]) - math.log(5000)) <= 1e-5 and (s.top_lp[1] + math.log(5000)).abs().max() <= 1e-5
    assert (s.top_lp[0, 5:] < -1e38).all()


def test_greedy_rows(torch, h):
    s = Set(torch, 4, 6000, 3, 4)
    s.temp[:] = torch.tensor([0.0, -1.0, 0.0, 0.5])
    s.logits[1, 100], s.logits[1, 4000] = 50.0, 50.0
    s.given[0, 0], s.given[1, 0], s.given[1, 1] = int(s.logits[0].argmax()), 100, 4000
    s.logits[2].fill_(-INF)
    h.logprobs(s.desc())
    s.check(torch)
    assert s.given_lp[1].tolist()[:2] == [0.0, -INF]


@pytest.mark.parametrize("t", [1e-30, 1e-38, 1e-6, 1e6, 1e38, 3e38, INF])
def test_extreme_temperatures(torch, h, t):
    """Toward 0 only the largest logits count, toward infinity all that are there alike."""
    import math
    s = Set(torch, 2, 3001, 2, 3, temp=True)
    s.temp.fill_(t)
    s.logits[1, 7], s.logits[1, 2000] = 60.0, 60.0
    s.logits[:, 100:103] = -INF
    s.given[:, 0], s.given[:, 1] = 7, 101
    h.logprobs(s.desc())
    assert (s.given_lp[:, 1] == -INF).all()
    if t < 1:
        assert abs(float(s.given_lp[1, 0]) + math.log(2)) <= 1e-6 and abs(float(s.entropy[1]) - math.log(2)) <= 1e-6
        assert float(s.entropy[0]) <= 1e-6 and abs(float(s.top_lp[0, 0])) <= 1e-6
    else:
        assert (s.entropy - math.log(2998)).abs().max() <= 1e-4 and (s.given_lp[:, 0] + math.log(2998)).abs().max() <= 1e-3


def test_nan_and_infinity(torch, h):
    """They make an ordinary row NaN and leave a greedy one; top lists what is larger than -infinity."""
    s = Set(torch, 5, 5000, 1, 3)
    s.given[:, 0] = 77
    s.logits[0, 4000] = NAN
    s.logits[1, 4000] = INF
    s.logits[2, 0] = NAN
    s.temp[2] = 0.0
    s.logits[3].fill_(-INF)
    s.logits[3, 4999] = NAN
    h.logprobs(s.desc())
    for r in (0, 1, 3):
        assert s.given_lp[r].isnan().all() and bool(s.entropy[r].isnan()) and s.top_lp[r].isnan().all()
    assert s.top[0].tolist() == plain.top(s.logits[0], 3) and s.top[1, 0] == 4000 and s.top[3].tolist() == [-1] * 3
    l = s.logits[2].cpu()
    assert s.top[2].tolist() == plain.top(l, 3) and s.top_lp[2].tolist() == [0.0, -INF, -INF] and float(s.entropy[2]) == 0.0
    s.check(torch, rows=[4])


def test_a_sharp_row_keeps_its_small_numbers(torch, h):
    """One likely token: its log probability and the entropy are near 0, and not lost in a difference."""
    s = Set(torch, 1, 4096, 1, 2, temp=False, std=1.0)
    s.logits[0, 1234] = 40.0
    s.given[0, 0] = 1234
    h.logprobs(s.desc())
    lp, H, _, _ = plain.logprobs(s.logits[0], 1.0)
    assert abs(float(s.given_lp[0, 0]) - float(lp[1234])) <= 1e-4 * abs(float(lp[1234])) and -1e-10 < float(lp[1234]) < 0
    assert abs(float(s.entropy[0]) - H) <= 1e-4 * H


def test_given_tokens_that_are_none(torch):
    with wt.Handle([]) as h:
        s = Set(torch, 2, 100, 3, 0)
        s.given.copy_(torch.tensor([[-1, 5, -2 ** 31], [6, 7, 8]]))
        h.logprobs(s.desc())
        s.check(torch)
        assert h.device_status() == 0
        s.given[1, 1] = 100
        h.logprobs(s.desc())
        torch.cuda.synchronize()
        assert h.device_status() == wt.WT_EINVAL and float(s.given_lp[1, 1]) == 0.0


def test_they_follow_from_probs(torch, h):
    """The two calls describe one distribution."""
    s = Set(torch, 3, 33333, 2, 9)
    p = torch.empty(3, 33333, device="cuda")
    h.probs(serving.probabilities(s.logits, p, temperature=s.temp))
    h.logprobs(s.desc())
    assert (p.gather(1, s.top.long()).log() - s.top_lp).abs().max() <= 1e-5
    assert (p.gather(1, s.given.long()).log() - s.given_lp).abs().max() <= 1e-5
    assert (-(p.double() * p.double().log()).sum(dim=1) - s.entropy).abs().max() <= 1e-4


def test_each_output_alone_and_repeatable(torch, h):
    s = Set(torch, 6, 70000, 2, 32)
    h.logprobs(s.desc())
    all_of = [t.clone() for t in (s.given_lp, s.entropy, s.top, s.top_lp)]
    for kw in (dict(given=None, given_lp=None), dict(entropy=None), dict(top=None, top_lp=None)):
        for t in (s.given_lp, s.entropy, s.top, s.top_lp):
            t.fill_(3)
        h.logprobs(s.desc(**kw))
        for t, w, name in zip((s.given_lp, s.entropy, s.top, s.top_lp), all_of, ("given", "entropy", "top", "top")):
            assert torch.equal(t, torch.full_like(t, 3) if name in kw else w), name
    for _ in range(20):  # whatever the timing
        h.logprobs(s.desc())
        assert all(torch.equal(a, b) for a, b in zip((s.given_lp, s.entropy, s.top, s.top_lp), all_of))


def test_in_a_graph(torch, h):
    s = Set(torch, 3, 20000, 1, 4)
    d, st = s.desc(), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        h.logprobs(d, torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        s.logits.normal_()
        g.replay()
        torch.cuda.synchronize()
        s.check(torch)


def test_what_is_refused(torch, h):
    def refuse(**kw):
        s = Set(torch, 3, 500, 2, 4)
        d = s.desc()
        for k, v in kw.items():
            setattr(d, k, v(d) if callable(v) else v)
        with pytest.raises(wt.WtError) as e:
            h.logprobs(d)
        assert e.value.code == wt.WT_EINVAL and "wt_logprobs" in str(e.value)

    for kw in (dict(rows=-1), dict(rows=1 << 28), dict(vocab=-1), dict(vocab=1 << 30, ldl=1 << 30), dict(ldl=499), dict(ldl=1 << 41),
               dict(n_given=-1), dict(n_given=3), dict(n_top=33), dict(n_top=-1), dict(given_stride=1), dict(logits=None),
               dict(given_lp=None), dict(top_lp=None), dict(logits=lambda d: d.logits + 2), dict(top=lambda d: d.logits + 80),
               dict(entropy=lambda d: d.temp), dict(entropy=lambda d: d.top), dict(given_lp=lambda d: d.given),
               dict(rows=1 << 20)):
        refuse(**kw)
    assert h.kernel_launches() == 0
    s = Set(torch, 3, 500, 2, 4)
    h.logprobs(s.desc(given=None, given_lp=None, entropy=None, top=None, top_lp=None))
    d = s.desc()
    d.rows = 0
    h.logprobs(d)
    assert h.kernel_launches() == 0
    for kw in (dict(given=s.given.long()), dict(given_lp=None), dict(top_lp=s.top_lp[:, :2]), dict(entropy=s.entropy[:2]),
               dict(temperature=s.temp.half()), dict(top=torch.zeros(3, 33, dtype=torch.int32, device="cuda"),
                                                     top_lp=torch.zeros(3, 33, device="cuda"))):
        with pytest.raises(ValueError):
            s.desc(**kw)


def test_an_empty_vocabulary(torch, h):
    """No token at all: as a row of -infinity alone."""
    s = Set(torch, 2, 1, 1, 2)
    d = s.desc()
    d.vocab, d.ldl = 0, 0
    s.given.fill_(-1)
    h.logprobs(d)
    assert s.given_lp.tolist() == [[0.0], [0.0]] and s.entropy.tolist() == [0.0, 0.0]
    assert s.top.tolist() == [[-1, -1]] * 2 and (s.top_lp == -INF).all()
