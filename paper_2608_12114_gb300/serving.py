"""Descriptors of a serving step's calls (include/wt_serve.h), made from torch tensors.

One step of several requests over one set of weights, beside Handle.pass_:

    h.pass_(...)                                   # projections, for every token of the step
    h.adapt([adapters(...), ...], stream)          # each request's low-rank adapter
    h.attend(attention(...), stream)               # over the shared prefix and the paged caches
    h.probs(probabilities(...), stream)            # the head's logits, at each row's temperature
    h.verify(verification(...), stream)            # which drafted tokens stay, and the next one

Each function here checks types, shapes and strides and returns the C descriptor, which holds the
tensors it points at; the values in them (lengths, slots, tokens) may change from step to step, so
a program makes its descriptors once and calls with them every step (wt.adapt_array keeps several
for one call).  PyTorch supplies device memory and streams only.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import wt

_TYPES = {torch.bfloat16: wt.WT_BF16, torch.float16: wt.WT_F16}


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _is(t, name: str, dtype, ndim: int):
    _need(isinstance(t, torch.Tensor) and t.is_cuda, "%s is a tensor in device memory" % name)
    _need(t.dtype == dtype and t.dim() == ndim, "%s is %d-dimensional %s, not %s of shape %s"
          % (name, ndim, dtype, t.dtype, tuple(t.shape)))


def _rows(t, name: str) -> int:
    """The pitch of a 2-D tensor whose rows are dense."""
    _need(t.stride(1) == 1 or t.shape[1] <= 1, "the rows of %s are contiguous" % name)
    if t.shape[0] <= 1:
        return max(1, t.shape[1])
    _need(t.stride(0) >= t.shape[1], "the rows of %s do not overlap" % name)
    return max(1, t.stride(0))


def _dense(t, name: str):
    _need(t.is_contiguous(), "%s is contiguous" % name)


def _ptr(t) -> Optional[int]:
    return None if t is None or t.numel() == 0 else t.data_ptr()


def adapters(x, y, slot, A, B, scale=None, rank=None, base=None) -> wt.AdaptDesc:
    """y[t] = base[t] + scale[s] B[s] (A[s] x[t]) with s = slot[t] (negative: no adapter).

    x [T, K] and the stacked factors A [S, R, K], B [S, M, R] are bf16 or f16; y and base [T, M] are
    fp32, base None adds to y in place.  slot int32 [T]; rank int32 [S] (None: R), scale fp32 [S]
    (None: 1)."""
    _need(x.dtype in _TYPES, "x is bf16 or f16, not %s" % x.dtype)
    _is(x, "x", x.dtype, 2), _is(A, "A", x.dtype, 3), _is(B, "B", x.dtype, 3)
    base = y if base is None else base
    _is(y, "y", torch.float32, 2), _is(base, "base", torch.float32, 2), _is(slot, "slot", torch.int32, 1)
    (T, K), (S, R, Ka), (Sb, M, Rb) = x.shape, A.shape, B.shape
    _need(Ka == K and Sb == S and Rb == R, "A [S, R, K] and B [S, M, R] fit x [T, K]: A %s, B %s, x %s"
          % (tuple(A.shape), tuple(B.shape), tuple(x.shape)))
    _need(tuple(y.shape) == (T, M) and tuple(base.shape) == (T, M) and tuple(slot.shape) == (T,),
          "y and base are [T, M] = [%d, %d] and slot is [T]" % (T, M))
    for t, name in ((rank, "rank"), (scale, "scale")):
        if t is not None:
            _is(t, name, torch.int32 if name == "rank" else torch.float32, 1), _dense(t, name)
            _need(t.shape[0] == S, "%s is [S]" % name)
    _dense(slot, "slot")
    for t, name, n in ((A, "A", R * K), (B, "B", M * R)):
        _need(S == 0 or n == 0 or t[0].is_contiguous(), "each slot of %s is contiguous" % name)
    d = wt.AdaptDesc(x=_ptr(x), base=_ptr(base), y=_ptr(y), slot=_ptr(slot), A=_ptr(A), B=_ptr(B), rank=_ptr(rank),
                     scale=_ptr(scale), ldx=_rows(x, "x"), ldbase=_rows(base, "base"), ldy=_rows(y, "y"),
                     a_slot=A.stride(0) if S > 1 else R * K, b_slot=B.stride(0) if S > 1 else M * R,
                     dtype=_TYPES[x.dtype], T=T, K=K, M=M, S=S, R=R)
    d.tensors = (x, base, y, slot, A, B, rank, scale)
    return d


def attention(q, out, begin, k_pages=None, v_pages=None, table=None, lens=None, *, max_new, max_len=0, prefix_k=None,
              prefix_v=None, scale=None) -> wt.AttendDesc:
    """Attention of each request's new tokens over a prefix all requests share and its own cache.

    q and out [tokens, heads, head_dim] (the heads of a token contiguous, any token pitch), bf16 or
    f16; begin int32 [requests + 1].  prefix_k, prefix_v [keys, kv_heads, head_dim], each key and head
    at any pitch (both tensors' alike).  k_pages, v_pages [pages, page, kv_heads, head_dim]; table
    int32 [requests, pages of a request]; lens int32 [requests], the new tokens' keys included.
    max_new and max_len bound what begin and lens will hold.  scale None: head_dim ** -0.5."""
    _need(q.dtype in _TYPES, "q is bf16 or f16, not %s" % q.dtype)
    _is(q, "q", q.dtype, 3), _is(out, "out", q.dtype, 3), _is(begin, "begin", torch.int32, 1)
    N, H, D = q.shape
    _need(out.shape == q.shape, "out has the shape of q")
    _need(begin.shape[0] >= 1, "begin is [requests + 1]")
    for t, name in ((q, "q"), (out, "out")):
        _need(N == 0 or t[0].is_contiguous(), "the heads of a token of %s are contiguous" % name)
    _dense(begin, "begin")
    n_req = begin.shape[0] - 1
    d = wt.AttendDesc(q=_ptr(q), out=_ptr(out), begin=_ptr(begin), dtype=_TYPES[q.dtype], n_req=n_req, n_tokens=N,
                      max_new=max_new, heads=H, head_dim=D, scale=D ** -0.5 if scale is None else scale,
                      q_stride=q.stride(0) if N > 1 else H * D, out_stride=out.stride(0) if N > 1 else H * D)
    Hkv = None
    _need((prefix_k is None) == (prefix_v is None), "prefix_k and prefix_v come together")
    if prefix_k is not None and prefix_k.shape[0]:
        _is(prefix_k, "prefix_k", q.dtype, 3), _is(prefix_v, "prefix_v", q.dtype, 3)
        P, Hkv, Dk = prefix_k.shape
        _need(Dk == D and prefix_v.shape == prefix_k.shape, "prefix_k and prefix_v are [keys, kv_heads, %d]" % D)
        # the stride of a dimension of one says nothing
        _need(all(n == 1 or a == b for n, a, b in zip(prefix_k.shape, prefix_k.stride(), prefix_v.stride())) and
              prefix_k.stride(2) == 1, "prefix_k and prefix_v have the same strides and contiguous head rows")
        d.prefix_k, d.prefix_v, d.prefix_len = _ptr(prefix_k), _ptr(prefix_v), P
        d.prefix_stride = prefix_k.stride(0) if P > 1 else Hkv * D
        d.prefix_head = prefix_k.stride(1) if Hkv > 1 else D
    if max_len:
        _is(k_pages, "k_pages", q.dtype, 4), _is(v_pages, "v_pages", q.dtype, 4)
        _is(table, "table", torch.int32, 2), _is(lens, "lens", torch.int32, 1)
        _dense(k_pages, "k_pages"), _dense(v_pages, "v_pages"), _dense(lens, "lens")
        n_pages, page, Hp, Dk = k_pages.shape
        _need(Dk == D and v_pages.shape == k_pages.shape and Hkv in (None, Hp),
              "k_pages and v_pages are [pages, page, kv_heads, %d], with the prefix's kv_heads" % D)
        _need(table.shape[0] == n_req and lens.shape[0] == n_req, "table and lens have a row for each request")
        Hkv = Hp
        d.k_pages, d.v_pages, d.table, d.len = _ptr(k_pages), _ptr(v_pages), _ptr(table), _ptr(lens)
        d.table_stride, d.page, d.n_pages, d.max_len = _rows(table, "table"), page, n_pages, max_len
        _need(max_len <= table.shape[1] * page, "max_len %d fits table's %d pages of %d" % (max_len, table.shape[1], page))
    d.kv_heads = H if Hkv is None else Hkv
    d.tensors = (q, out, begin, prefix_k, prefix_v, k_pages, v_pages, table, lens)
    return d


def probabilities(logits, p, temperature=None) -> wt.ProbsDesc:
    """p[r] = softmax(logits[r] / temperature[r]); a temperature of 0 takes the first largest logit.
    logits and p fp32 [rows, vocab] (p may be logits), temperature fp32 [rows] (None: 1)."""
    _is(logits, "logits", torch.float32, 2), _is(p, "p", torch.float32, 2)
    _need(p.shape == logits.shape, "p has the shape of logits")
    if temperature is not None:
        _is(temperature, "temperature", torch.float32, 1), _dense(temperature, "temperature")
        _need(temperature.shape[0] == logits.shape[0], "temperature is [rows]")
    d = wt.ProbsDesc(logits=_ptr(logits), p=_ptr(p), temp=_ptr(temperature), ldl=_rows(logits, "logits"),
                     ldp=_rows(p, "p"), rows=logits.shape[0], vocab=logits.shape[1])
    d.tensors = (logits, p, temperature)
    return d


def verification(p, drafted, begin, u, u_draw, accepted, tokens, q=None) -> wt.VerifyDesc:
    """Drafted tokens against the target's probabilities (see wt_verify).

    p fp32 [drafted + requests, vocab], q fp32 [drafted, vocab] or None (certain drafts), drafted
    int32 [n], begin int32 [requests + 1], u fp32 [n], u_draw fp32 [requests]; outputs accepted int32
    [requests], tokens int32 [requests, longest draft + 1]."""
    _is(p, "p", torch.float32, 2), _is(drafted, "drafted", torch.int32, 1), _is(begin, "begin", torch.int32, 1)
    _is(u, "u", torch.float32, 1), _is(u_draw, "u_draw", torch.float32, 1)
    _is(accepted, "accepted", torch.int32, 1), _is(tokens, "tokens", torch.int32, 2)
    for t, name in ((drafted, "drafted"), (begin, "begin"), (u, "u"), (u_draw, "u_draw"), (accepted, "accepted"),
                    (tokens, "tokens")):
        _dense(t, name)
    n, B, V = drafted.shape[0], accepted.shape[0], p.shape[1]
    _need(p.shape[0] == n + B, "p has a row for each drafted token and one more for each request")
    _need(begin.shape[0] == B + 1 and u.shape[0] == n and u_draw.shape[0] == B and tokens.shape[0] == B and
          tokens.shape[1] >= 1, "begin is [requests + 1], u [drafted], u_draw [requests], tokens [requests, longest + 1]")
    if q is not None:
        _is(q, "q", torch.float32, 2)
        _need(tuple(q.shape) == (n, V), "q is [drafted, vocab]")
    # an empty q still says that drafts were not certain; it is then never read
    d = wt.VerifyDesc(p=_ptr(p), q=None if q is None else q.data_ptr() or _ptr(p), drafted=_ptr(drafted), begin=_ptr(begin),
                      u=_ptr(u), u_draw=_ptr(u_draw), accepted=_ptr(accepted), tokens=_ptr(tokens), ldp=_rows(p, "p"),
                      ldq=V if q is None else _rows(q, "q"), n_req=B, n_drafted=n, max_draft=tokens.shape[1] - 1, vocab=V)
    d.tensors = (p, drafted, begin, u, u_draw, accepted, tokens, q)
    return d
