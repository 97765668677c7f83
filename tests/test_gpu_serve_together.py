"""A step through placing, both kinds of attention and log probabilities: one after another as a program makes
them, in a graph, from threads and on many streams."""
import ctypes as C
import threading

import pytest

from paper_2608_12114_gb300 import build, serving, wt
from tests import _serve, _serve_more as plain
from tests import test_gpu_serve_cross, test_gpu_serve_logprobs, test_gpu_serve_place

pytestmark = pytest.mark.gpu
Cross, Logprobs, Place = test_gpu_serve_cross.Set, test_gpu_serve_logprobs.Set, test_gpu_serve_place.Set


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


class Layer:
    """Attention of a decoder's layer with an encoder behind it, and the head's logits: new tokens of three
    requests, their caches, their memories."""

    H, HKV, D, V = 8, 2, 64, 3001

    def __init__(self, torch, seed=0):
        self.s = Place(torch, [4, 1, 3], [20, 55, 0], H=self.H, Hkv=self.HKV, D=self.D, norm="bf16", seed=seed)
        self.mem = Cross(torch, [4, 1, 3], [200, 77, 513], self.H, self.HKV, self.D, holes=0.2, seed=seed)
        g = torch.Generator("cuda").manual_seed(seed)
        N = 8
        self.w = torch.randn(self.H * self.D, self.V, device="cuda", generator=g) / 4
        self.own, self.cross_q = torch.empty_like(self.s.q_out), torch.empty_like(self.s.q_out)
        self.logits = torch.empty(N, self.V, device="cuda")
        self.given = torch.randint(0, self.V, (N, 1), device="cuda", generator=g).int()
        self.lp, self.ent = torch.empty(N, 1, device="cuda"), torch.empty(N, device="cuda")
        s, m = self.s, self.mem
        m.out = torch.empty_like(s.q_out)
        self.calls = (s.desc(),
                      serving.attention(s.q_out, self.own, s.begin, s.k_pages, s.v_pages, s.table, s.lens, max_new=4, max_len=s.max_len),
                      serving.placement(q=self.own, q_out=self.cross_q, q_norm=s.q_norm),
                      serving.cross_attention(self.cross_q, m.out, s.begin, m.k, m.v, m.mem_begin, m.mem_len, max_new=4, max_mem=513,
                                              keep=m.keep),
                      serving.log_probabilities(self.logits, given=self.given, given_lp=self.lp, entropy=self.ent))

    def run(self, torch, h, stream):
        for call, d in zip((h.place, h.attend, h.place, h.cross), self.calls):
            call(d, stream)
        torch.mm(self.mem.out.view(8, -1).float(), self.w, out=self.logits)
        h.logprobs(self.calls[4], stream)

    def check(self, torch):
        """Each call against 64 bits on what it was given."""
        s, m = self.s, self.mem
        s.check(torch)
        D = self.D
        for got, (want, mag, qk) in (
                (self.own, _serve.attend(s.q_out, s.begin, None, None, s.k_pages, s.v_pages, s.table, s.lens, D ** -0.5)),
                (m.out, plain.cross(self.cross_q, s.begin, m.k, m.v, m.mem_begin, m.mem_len, m.keep, D ** -0.5))):
            tol = (2.0 ** -8 + 2 * (D / 16 + 4) * 2.0 ** -23 * qk + 2.0 ** -15) * mag + 2.0 ** -8 * want.abs()
            assert ((got.double().cpu() - want).abs() <= tol).all()
        for t in range(8):
            y, mag = plain.place_head(self.own[t].cpu(), s.q_norm.cpu(), 1e-6, [], [], False)
            assert ((self.cross_q[t].double().cpu() - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -19 * mag).all()
            lp, H, m1, m2 = plain.logprobs(self.logits[t], 1.0)
            tol = 2.0 ** -20 * (1 + m1 + m2 + abs(float(lp[int(self.given[t])])))
            assert abs(float(self.lp[t]) - float(lp[int(self.given[t])])) <= tol and abs(float(self.ent[t]) - H) <= tol


def test_a_step_of_a_layer(torch, h):
    a = Layer(torch)
    a.run(torch, h, 0)
    a.check(torch)


def test_a_step_in_a_graph(torch, h):
    """Captured without a step before it; replayed with other rows, fewer keys and shorter memories."""
    a, st = Layer(torch), torch.cuda.Stream()
    torch.mm(a.mem.out.view(8, -1).float(), a.w, out=a.logits)  # the library's own workspaces
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        a.run(torch, h, torch.cuda.current_stream().cuda_stream)
    for step in range(3):
        for t in (a.s.q, a.s.k, a.s.v):
            t.normal_()
        a.s.lens -= torch.tensor([step, step, 0], dtype=torch.int32, device="cuda")
        a.mem.mem_len[1] = 77 - 30 * step
        a.s.before = [t.clone() for t in (a.s.q_out, a.s.k_pages, a.s.v_pages)]
        g.replay()
        torch.cuda.synchronize()
        a.check(torch)


def test_threads_and_streams(torch, h):
    """Two threads on one handle, then eleven streams at once, each with its step."""
    layers = [Layer(torch, seed=i) for i in range(11)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    failed = []

    def body(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(30):
                    layers[i].run(torch, h, streams[i].cuda_stream)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=body, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(11):
            with torch.cuda.stream(streams[i]):
                layers[i].run(torch, h, streams[i].cuda_stream)
    torch.cuda.synchronize()
    assert not failed
    for a in layers:
        a.check(torch)


def test_calls_of_different_sizes_share_a_stream(torch, h):
    """Their workspaces are one; each call's kernels wait for those of the call before."""
    sets = [Cross(torch, [1], [1500], 32, 8, 128), Cross(torch, [300, 70], [500, 1000], 8, 4, 64), Cross(torch, [5] * 3, [99, 0, 700], 8, 8, 80),
            Logprobs(torch, 40, 30000, 1, 20), Logprobs(torch, 3, 128256, 1, 32), Logprobs(torch, 900, 1000, 2, 0)]
    descs = [s.desc() for s in sets]
    for _ in range(20):
        for s, d in zip(sets, descs):
            (h.cross if isinstance(s, Cross) else h.logprobs)(d)
    for s in sets:
        if isinstance(s, Cross):
            s.check(torch)
        else:
            s.check(torch, rows=range(0, len(s.logits), max(1, len(s.logits) // 8)))


def test_the_first_kernel_of_a_call_waits_for_the_stream(torch, h):
    """In a capture, the edge to a call's first kernel from what came before it is a full one."""
    rt = C.CDLL("libcudart.so.13")
    rt.cudaStreamBeginCapture.argtypes = [C.c_void_p, C.c_int]
    rt.cudaStreamEndCapture.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
    rt.cudaGraphGetEdges.argtypes = [C.c_void_p] + [C.c_void_p] * 4
    rt.cudaGraphDestroy.argtypes = [C.c_void_p]
    few, many, lp = Cross(torch, [1], [1500], 8, 2, 64), Cross(torch, [300], [500], 8, 4, 64), Logprobs(torch, 3, 128256, 1, 32)
    d = [few.desc(), many.desc(), lp.desc(), Place(torch, [2], [3]).desc()]
    calls = [lambda st: h.cross(d[0], st), lambda st: h.cross(d[1], st), lambda st: h.logprobs(d[2], st), lambda st: h.place(d[3], st)]
    mark, st = torch.zeros(4, device="cuda"), torch.cuda.Stream()
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
        assert [data[8 * i + 2] for i in range(n.value) if frm[i] in first] == [0]
        rt.cudaGraphDestroy(g)


def test_the_example_gives_log_probabilities(torch, tmp_path):
    import os
    import sys

    from paper_2608_12114_gb300 import synth
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        import serving_step as ex
    finally:
        sys.path.pop(0)
    ck = synth.build("mid", str(tmp_path), layers=1, vocab=1024)
    with wt.Handle(ck.paths) as h:
        m = ex.Decoder(h)
        a = ex.inputs(1024, ex.HEADS * ex.DIM)
        r = ex.step(m, **a)
        torch.cuda.synchronize()
        assert h.device_status() == 0
        of = torch.repeat_interleave(torch.arange(3), a["begin"].diff().cpu().long())
        for t in range(len(of)):
            temp = float(a["temperature"][of[t]])
            lp, H, m1, m2 = plain.logprobs(r["logits"][t], temp)
            v = int(r["given"][t])
            want = 0.0 if v < 0 else float(lp[v])
            got = float(r["lp"][t])
            assert got == want if want in (0.0, -plain.INF) else abs(got - want) <= 2.0 ** -20 * (1 + m1 + abs(want))
            assert r["top"][t].tolist() == plain.top(r["logits"][t].cpu(), 5)
