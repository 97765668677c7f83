"""How a program makes the serving calls: from threads and streams, into graphs, many at a time, again and again."""
import ctypes as C
import gc
import os
import subprocess
import sys
import threading
import time

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


def test_the_first_kernel_of_a_call_waits_for_the_stream(torch, h):
    """In a capture, the edge to a call's first kernel from what came before it is a full one: only the
    kernels within a call follow one another programmatically."""
    rt = C.CDLL("libcudart.so.13")
    rt.cudaStreamBeginCapture.argtypes = [C.c_void_p, C.c_int]
    rt.cudaStreamEndCapture.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
    rt.cudaGraphGetEdges.argtypes = [C.c_void_p] + [C.c_void_p] * 4
    rt.cudaGraphDestroy.argtypes = [C.c_void_p]
    x = make(torch, 300, 64, 32, 2, 8, torch.bfloat16)
    sets = [Set(torch, [2, 1], None, 0, 4, 2, 64), Set(torch, [2, 1], [40, 33], 0, 4, 2, 64), Set(torch, [2, 1], [40, 33], 900, 4, 2, 64),
            Set(torch, [2] * 20, [9] * 20, 900, 4, 2, 64), Set(torch, [2] * 20, None, 900, 4, 2, 64)]
    calls = [lambda st, s=s: h.attend(s.desc(), st) for s in sets]  # the first: no key at all
    calls.append(lambda st: h.adapt([serving.adapters(x[0], x[1], x[2], x[3], x[4], x[5], base=x[6])], st))
    mark = torch.zeros(4, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call in calls:
        g, n = C.c_void_p(), C.c_size_t()
        assert rt.cudaStreamBeginCapture(st.cuda_stream, 2) == 0
        try:
            with torch.cuda.stream(st):
                mark.fill_(1.0)
            call(st.cuda_stream)
        finally:
            assert rt.cudaStreamEndCapture(st.cuda_stream, C.byref(g)) == 0
        assert rt.cudaGraphGetEdges(g, None, None, None, C.byref(n)) == 0 and n.value >= 1
        frm, to, data = (C.c_void_p * n.value)(), (C.c_void_p * n.value)(), (C.c_uint8 * (8 * n.value))()
        assert rt.cudaGraphGetEdges(g, frm, to, data, C.byref(n)) == 0
        first = set(frm) - set(to)
        assert len(first) == 1
        kinds = [data[8 * i + 2] for i in range(n.value) if frm[i] in first]
        assert kinds == [0], kinds
        rt.cudaGraphDestroy(g)


def test_threads_on_one_handle(torch, h):
    """Two threads, each with its stream, its calls of every kind and its sizes."""
    sets = [Set(torch, [1 + i] * 6, [40] * 6, 900 + 700 * i, 8, 2, 128, seed=i) for i in range(2)]
    ads = [make(torch, 280 + 40 * i, 96, 64, 3, 16, torch.float16, seed=i) for i in range(2)]
    wants = [s.want() for s in sets]
    wad = [_serve.adapt(x, s, A, B, c, None, b) for x, y, s, A, B, c, b in ads]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    failed = []

    def body(i):
        try:
            x, y, s, A, B, c, b = ads[i]
            da, dd = sets[i].desc(), [serving.adapters(x, y, s, A, B, c, base=b)]
            for _ in range(200):
                h.attend(da, streams[i].cuda_stream)
                h.adapt(dd, streams[i].cuda_stream)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=body, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for i in range(2):
        sets[i].check(torch, wants[i])
        close(torch, ads[i][1], wad[i], 96, 16)


def test_the_first_call_of_a_thread_is_checked(torch, h):
    """Before any other use of the GPU on it: the range of every buffer, as on other threads."""
    torch.cuda.empty_cache()
    l, p = (torch.zeros(8, 1 << 20, device="cuda") for _ in range(2))  # allocations of their own
    d = serving.probabilities(l, p)
    d.rows = 1 << 16
    got = []
    t = threading.Thread(target=lambda: got.append((wt.lib().wt_probs(h.ptr, C.byref(d), None), wt.lib().wt_last_error())))
    t.start()
    t.join()
    assert got[0][0] == wt.WT_EINVAL and b"runs past" in got[0][1]


SECOND = 2_000_000_000  # cycles, about


def test_a_larger_call_does_not_wait_for_the_stream(torch, h):
    """Its stream is busy for a second with work the smaller call's workspace waits for."""
    a, b = Set(torch, [1], [60], 2000, 8, 2, 128), Set(torch, [2] * 30, [60] * 30, 4000, 8, 2, 128)
    other = torch.cuda.Stream()
    with wt.Handle([]) as warm:
        warm.attend(b.desc()), warm.attend(a.desc())
        torch.cuda.synchronize()
    wa, wb = a.want(), b.want()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        torch.cuda._sleep(SECOND)
        t0 = time.perf_counter()
        h.attend(a.desc(), other.cuda_stream)
        h.attend(b.desc(), other.cuda_stream)
        took, busy = time.perf_counter() - t0, not other.query()
    assert busy and took < 0.2, took
    other.synchronize()
    a.check(torch, wa), b.check(torch, wb)
    h.attend(a.desc(), other.cuda_stream)
    other.synchronize()
    a.check(torch, wa)


def test_many_streams_do_not_wait_for_one_another(torch, h):
    s = Set(torch, [1] * 8, [60] * 8, 2000, 8, 2, 128)
    want = s.want()
    h.attend(s.desc())
    streams = [torch.cuda.Stream() for _ in range(20)]
    torch.cuda.synchronize()
    for st in streams[:1]:
        with torch.cuda.stream(st):
            torch.cuda._sleep(SECOND)
    t0 = time.perf_counter()
    for st in streams:
        h.attend(s.desc(), st.cuda_stream)
    took, busy = time.perf_counter() - t0, not streams[0].query()
    assert busy and took < 0.3, took
    torch.cuda.synchronize()
    s.check(torch, want)
    # finished streams' workspaces serve later ones: no more of them however many streams come
    before = wt.live()["device_bytes"]
    for _ in range(40):
        st = torch.cuda.Stream()
        h.attend(s.desc(), st.cuda_stream)
        st.synchronize()
    assert wt.live()["device_bytes"] == before



def capturing(torch, mode):
    """A capture open on another thread: (start it, end it and say whether it held)."""
    begun, end, ok = threading.Event(), threading.Event(), []

    def body():
        st, x = torch.cuda.Stream(), torch.zeros(8, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        try:
            with torch.cuda.stream(st):
                g.capture_begin(capture_error_mode=mode)
                x += 1
                begun.set()
                end.wait(60)
                x += 1
                g.capture_end()
            g.replay()
            torch.cuda.synchronize()
            ok.append(x.tolist() == [2.0] * 8)
        except Exception as e:
            ok.append(str(e))
        finally:
            begun.set()

    t = threading.Thread(target=body)
    t.start()
    begun.wait(60)

    def finish():
        end.set()
        t.join(60)
        return ok

    return finish


@pytest.mark.parametrize("mode", ["global", "thread_local"])
def test_a_handle_used_and_closed_while_another_thread_captures(torch, mode):
    p, q, d, begin, u, w = drafts(torch, [3, 0, 2], 5003, 2.0, False)
    acc, tok = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    a = Set(torch, [1] * 8, [60] * 8, 2000, 8, 2, 128)
    want, wa = _serve.verify(p, q, d, begin, u, w, 3), a.want()
    desc, da = serving.verification(p, d, begin, u, w, acc, tok, q=q), a.desc()
    st = torch.cuda.Stream()
    h = wt.Handle([])
    torch.cuda.synchronize()
    finish = capturing(torch, mode)
    try:
        h.verify(desc, st.cuda_stream)
        h.attend(da, st.cuda_stream)
        h.close()
    finally:
        ok = finish()
    assert ok == [True]
    torch.cuda.synchronize()
    assert (acc.tolist(), tok.tolist()) == want
    a.check(torch, wa)


FIRST = """
import sys, torch
from paper_2608_12114_gb300 import serving, wt
from tests.test_gpu_serve_adapt import make
from tests.test_gpu_serve_attend import Set
from tests.test_gpu_serve_draw import drafts
x, y, slot, A, B, scale, base = make(torch, 300, 64, 32, 2, 8, torch.bfloat16)
s = Set(torch, [2] * 20, [9] * 20, 900, 4, 2, 64)
l, p = torch.randn(3, 50021, device="cuda"), torch.empty(3, 50021, device="cuda")
v = drafts(torch, [2, 1], 500, 1.0, False)
acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
ds = dict(adapt=[serving.adapters(x, y, slot, A, B, scale, base=base)], attend=s.desc(), probs=serving.probabilities(l, p),
          verify=serving.verification(v[0], v[2], v[3], v[4], v[5], acc, tok, q=v[1]))
outs = (y, s.out, p, acc, tok)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with wt.Handle([]) as h:
    with torch.cuda.graph(g):
        for name, d in ds.items():
            getattr(h, name)(d, torch.cuda.current_stream().cuda_stream)
    g.replay()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    for name, d in ds.items():
        getattr(h, name)(d)
    torch.cuda.synchronize()
    assert h.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(first, outs)) and not any(torch.isnan(t.float()).any() for t in outs)
print("same")
"""


def test_the_first_calls_of_a_process_may_be_captured(torch):
    """No warm-up: kernels are loaded and made ready inside the capture."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stderr[-2000:]


def test_an_array_of_descriptors_keeps_its_tensors(torch, h):
    x, y, slot, A, B, scale, base = make(torch, 12, 64, 40, 3, 8, torch.bfloat16)
    want = _serve.adapt(x, slot, A, B, scale, None, base)

    def step():
        y2 = [y.clone(), y.clone()]
        a = wt.adapt_array([serving.adapters(x.clone(), t, slot.clone(), A.clone(), B.clone(), scale.clone(), base=base.clone())
                            for t in y2])
        return a, y2

    a, ys = step()
    gc.collect()
    junk = [torch.full((1 << 16,), _serve.NAN, device="cuda") for _ in range(64)]
    h.adapt(a)
    torch.cuda.synchronize()
    assert len(a) == 2 and len(junk) == 64
    for t in ys:
        close(torch, t, want, 64, 8)


def test_the_order_of_projections_changes_nothing(torch, h):
    """A launch's clusters, and with them the order of the sums, go by all its projections, not by the first."""
    sets = [make(torch, T, 512, 64, S, 64, torch.bfloat16, seed=T) for T, S in ((1, 1), (250, 20))]

    def call(order):
        for i in order:
            sets[i][1].fill_(_serve.NAN)
        h.adapt([serving.adapters(x, y, s, A, B, c, base=b) for x, y, s, A, B, c, b in (sets[i] for i in order)])
        torch.cuda.synchronize()
        return [sets[i][1].clone() for i in (0, 1)]

    for a, b in zip(call((0, 1)), call((1, 0))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["bfloat16", "float16"])
def test_many_tokens_through_many_projections(torch, h, dt):
    """More projections than a launch takes, of several slot maps, lengths and ranks, some in place."""
    sets = []
    for i in range(11):
        T = (300, 300, 270, 5)[i % 4]
        x, y, slot, A, B, scale, base = make(torch, T, 72 + 8 * i, 50 + i, 3 + i % 2, 1 + 5 * i, getattr(torch, dt), seed=i)
        if i % 4 == 1:  # the map of the one before
            slot = sets[-1][2] if sets[-1][3].shape[0] >= A.shape[0] else slot
        if i % 3 == 2:
            y = base.clone()
        sets.append((x, y, slot, A, B, scale, base, i % 3 == 2))
    want = [_serve.adapt(x, s, A, B, c, None, b) for x, y, s, A, B, c, b, _ in sets]
    for _ in range(2):
        for x, y, s, A, B, c, b, inplace in sets:
            y.copy_(b) if inplace else y.fill_(_serve.NAN)
        h.adapt([serving.adapters(x, y, s, A, B, c, base=None if inplace else b) for x, y, s, A, B, c, b, inplace in sets])
        torch.cuda.synchronize()
        for (x, y, s, A, B, c, b, _), r in zip(sets, want):
            close(torch, y, r, x.shape[1], A.shape[1])


def test_a_batch_that_takes_small_clusters(torch, h):
    """48 tokens of 32 slots through three projections: A x is split otherwise than for one token, so bits
    may differ, but no more than the order of the sums."""
    sets = [make(torch, 48, 512, M, 32, 32, torch.bfloat16, seed=3) for M in (256, 64, 64)]
    x, _, slot, _, _, _, _ = sets[0]
    descs = [serving.adapters(x, y, slot, A, B, c, base=b) for _, y, _, A, B, c, b in sets]
    h.adapt(descs)
    torch.cuda.synchronize()
    for _, y, _, A, B, c, b in sets:
        want = _serve.adapt(x, slot, A, B, c, None, b)
        close(torch, y, want, 512, 32)
        one = torch.full_like(y, _serve.NAN)
        for t in range(48):
            h.adapt([serving.adapters(x[t:t + 1], one[t:t + 1], slot[t:t + 1], A, B, c, base=b[t:t + 1])])
        torch.cuda.synchronize()
        close(torch, one, want, 512, 32)


@pytest.mark.parametrize("new,lens,P", [([300], [300], 0), ([257, 1, 190], [400, 9, 190], 0), ([200, 150], [210, 150], 140)])
def test_prompts(torch, h, new, lens, P):
    s = Set(torch, new, lens, P, 4, 2, 64)
    want = s.want()
    h.attend(s.desc())
    torch.cuda.synchronize()
    s.check(torch, want)


@pytest.mark.parametrize("new,lens,P", [([1], [37], 500), ([1] * 24, [900 - 30 * i for i in range(24)], 6000), ([3] * 20, [200] * 20, 3000)])
def test_calls_repeat_themselves(torch, h, new, lens, P):
    s = Set(torch, new, lens, P, 8, 2, 128)
    h.attend(s.desc())
    first = s.out.clone()
    for _ in range(30):
        s.out.fill_(_serve.NAN)
        h.attend(s.desc())
        assert torch.equal(s.out, first)


def test_a_later_draft_changes_nothing_before_it(torch, h):
    s = Set(torch, [6], [50], 40, 4, 2, 64)
    h.attend(s.desc())
    first, k, v = s.out.clone(), s.k.clone(), s.v.clone()
    for j in range(45, 50):
        s.k.copy_(k), s.v.copy_(v)
        at = s.table[0, j // 16]
        s.k[at, j % 16], s.v[at, j % 16] = 3.0, -5.0
        h.attend(s.desc())
        torch.cuda.synchronize()
        assert torch.equal(s.out[:j - 44], first[:j - 44])
        assert not torch.equal(s.out[j - 44:], first[j - 44:])
