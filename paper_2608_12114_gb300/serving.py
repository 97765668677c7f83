"""Descriptors of a serving step's calls (include/wt_serve.h), made from torch tensors.

One step of several requests over one set of weights, beside Handle.pass_:

    h.pass_(...)                                   # projections, for every token of the step
    h.adapt([adapters(...), ...], stream)          # each request's low-rank adapter
    h.place(placement(...), stream)                # norms, rotation; keys and values to their pages
    h.attend(attention(...), stream)               # over the shared prefix and the paged caches
    h.cross(cross_attention(...), stream)          # to each request's memory, as an encoder's states
    h.probs(probabilities(...), stream)            # the head's logits, at each row's temperature
    h.logprobs(log_probabilities(...), stream)     # of given tokens, with entropy and alternatives
    h.verify(verification(...), stream)            # which drafted tokens stay, and the next one

Each function here checks types, shapes and strides and returns the C descriptor, which holds the
tensors it points at; the values in them (lengths, slots, tokens) may change from step to step, so
a program makes its descriptors once and calls with them every step (wt.adapt_array keeps several
for one call).  PyTorch supplies device memory and streams only.
"""
from __future__ import annotations

import math
from fractions import Fraction
from typing import Optional, Sequence

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


_PI = Fraction(31415926535897932384626433832795028841971, 10 ** 40)  # off by less than 2^-132


def turns(freq: Sequence[float], device="cuda") -> torch.Tensor:
    """For placement: the turns that a position adds for each pair, modulo one, as 64-bit fractions (int64
    bits).  freq holds radians a position, as floats in 64 bits; the quotient by 2 pi is rounded once."""
    v = []
    for f in freq:
        _need(math.isfinite(f), "freq is finite")
        t = round(Fraction(f) * 2 ** 63 / _PI) % 2 ** 64
        v.append(t - 2 ** 64 if t >= 2 ** 63 else t)
    return torch.tensor(v, dtype=torch.int64, device=device)


def placement(begin=None, k_pages=None, v_pages=None, table=None, lens=None, *, q=None, q_out=None, k=None, v=None, max_len=0,
              q_norm=None, k_norm=None, eps=1e-6, turns=None, axis=None, pos=None, first_pos=0,
              neighbours=False) -> wt.PlaceDesc:
    """Queries to q_out, keys and values to their requests' pages, normed and rotated on the way (see wt_place).

    q [tokens, heads, head_dim] and k, v [tokens, kv_heads, head_dim] (the heads of a token contiguous, any
    token pitch) are fp32 or of the outputs' type, bf16 or f16; any of them may be None.  q_out has q's shape.
    begin, the pages, table, lens and max_len are attention's.  q_norm, k_norm [head_dim] (None: no norm).
    turns (of serving.turns) rotates the first 2 len(turns) elements of each head, by the token's place plus
    first_pos, or by pos int32 [tokens, axes], pair j by its axis[j] (None: all by the first)."""
    _need(q is not None or k is not None or v is not None, "one of q, k and v at least")
    _need((q is None) == (q_out is None), "q and q_out come together")
    _need(k is None or k_pages is not None, "k goes with k_pages")
    _need(v is None or v_pages is not None, "v goes with v_pages")
    out = q_out if q is not None else k_pages if k is not None else v_pages
    _need(out.dtype in _TYPES, "q_out and the pages are bf16 or f16, not %s" % out.dtype)
    src = q if q is not None else k if k is not None else v
    _need(src.dtype in (torch.float32, out.dtype), "q, k and v are fp32 or %s, not %s" % (out.dtype, src.dtype))
    N, D = src.shape[0], src.shape[-1]
    d = wt.PlaceDesc(in_dtype=wt.WT_F32 if src.dtype == torch.float32 else _TYPES[out.dtype], dtype=_TYPES[out.dtype],
                     n_tokens=N, head_dim=D, eps=eps, first_pos=first_pos, flags=wt.WT_PLACE_NEIGHBOURS if neighbours else 0)
    Hkv = None
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if t is None:
            continue
        _is(t, name, src.dtype, 3)
        _need(t.shape[0] == N and t.shape[2] == D, "%s is [%d, heads, %d]" % (name, N, D))
        _need(N == 0 or t[0].is_contiguous(), "the heads of a token of %s are contiguous" % name)
        setattr(d, name, _ptr(t))
        setattr(d, name + "_stride", t.stride(0) if N > 1 else t.shape[1] * D)
        if name != "q":
            _need(Hkv in (None, t.shape[1]), "k and v have as many heads")
            Hkv = t.shape[1]
    if q is not None:
        _is(q_out, "q_out", out.dtype, 3)
        _need(q_out.shape == q.shape, "q_out has the shape of q")
        _need(N == 0 or q_out[0].is_contiguous(), "the heads of a token of q_out are contiguous")
        d.q_out, d.heads, d.out_stride = _ptr(q_out), q.shape[1], q_out.stride(0) if N > 1 else q.shape[1] * D
    norm = q_norm if q_norm is not None else k_norm
    for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None:
            _need(t.dtype in (torch.float32, torch.bfloat16, torch.float16), "%s is fp32, bf16 or f16, not %s" % (name, t.dtype))
            _is(t, name, norm.dtype, 1), _dense(t, name)
            _need(t.shape[0] == D, "%s is [%d]" % (name, D))
            setattr(d, name, _ptr(t))
            d.norm_dtype = wt.WT_F32 if t.dtype == torch.float32 else _TYPES[t.dtype]
    if begin is not None:
        _is(begin, "begin", torch.int32, 1), _dense(begin, "begin")
        _need(begin.shape[0] >= 1, "begin is [requests + 1]")
        d.begin, d.n_req = _ptr(begin), begin.shape[0] - 1
    if lens is not None:
        _is(lens, "lens", torch.int32, 1), _dense(lens, "lens")
        _need(begin is not None and lens.shape[0] == d.n_req, "lens has a row for each request")
        _need(max_len >= 1, "max_len bounds what lens will hold")
        d.len, d.max_len = _ptr(lens), max_len
    if Hkv is not None:
        _need(begin is not None and table is not None and lens is not None, "k and v go with begin, table and lens")
        _is(table, "table", torch.int32, 2)
        _need(table.shape[0] == d.n_req, "table has a row for each request")
        shape = None
        for t, p, name in ((k, k_pages, "k_pages"), (v, v_pages, "v_pages")):
            if t is None:
                continue
            _is(p, name, out.dtype, 4), _dense(p, name)
            _need(p.shape[2:] == (Hkv, D) and shape in (None, p.shape), "k_pages and v_pages are [pages, page, %d, %d]" % (Hkv, D))
            shape = p.shape
            setattr(d, name, _ptr(p))
        d.kv_heads, d.n_pages, d.page = Hkv, shape[0], shape[1]
        d.table, d.table_stride = _ptr(table), _rows(table, "table")
        _need(max_len <= table.shape[1] * d.page, "max_len %d fits table's %d pages of %d" % (max_len, table.shape[1], d.page))
    if turns is not None:
        _is(turns, "turns", torch.int64, 1), _dense(turns, "turns")
        d.turns, d.rot_dim = _ptr(turns), 2 * turns.shape[0]
        _need(d.rot_dim <= D and d.rot_dim % 8 == 0, "turns are for a multiple of 4 pairs of a head's %d elements" % D)
        if pos is not None:
            _is(pos, "pos", torch.int32, 2)
            _need(pos.shape[0] == N and 1 <= pos.shape[1] <= wt.WT_PLACE_MAX_AXES, "pos is [%d, up to %d axes]" % (N, wt.WT_PLACE_MAX_AXES))
            d.pos, d.pos_stride, d.axes = _ptr(pos), _rows(pos, "pos"), pos.shape[1]
            if axis is not None:
                _need(len(axis) == turns.shape[0] and all(0 <= a < d.axes for a in axis), "axis has one of %d for each pair" % d.axes)
                d.axis[:len(axis)] = [int(a) for a in axis]
        else:
            _need(axis is None, "axis goes with pos")
            _need(begin is not None and lens is not None, "tokens without pos have a place by begin and lens")
    else:
        _need(pos is None and axis is None, "pos and axis go with turns")
    d.tensors = (q, q_out, k, v, q_norm, k_norm, begin, k_pages, v_pages, table, lens, turns, pos)
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


def cross_attention(q, out, begin, k, v, mem_begin, mem_len, *, max_new, max_mem, keep=None, scale=None) -> wt.CrossDesc:
    """Attention of each request's tokens to a memory of its own (see wt_cross).

    q, out and begin are attention's.  k and v [states, kv_heads, head_dim], of q's type, each state and head
    at any pitch (both tensors' alike); mem_begin and mem_len int32 [requests].  keep uint8 [states] (None:
    all).  max_new and max_mem bound what begin and mem_len will hold.  scale None: head_dim ** -0.5."""
    _need(q.dtype in _TYPES, "q is bf16 or f16, not %s" % q.dtype)
    _is(q, "q", q.dtype, 3), _is(out, "out", q.dtype, 3), _is(k, "k", q.dtype, 3), _is(v, "v", q.dtype, 3)
    N, H, D = q.shape
    M, Hkv, Dk = k.shape
    _need(out.shape == q.shape, "out has the shape of q")
    _need(Dk == D and v.shape == k.shape, "k and v are [states, kv_heads, %d]" % D)
    for t, name in ((q, "q"), (out, "out")):
        _need(N == 0 or t[0].is_contiguous(), "the heads of a token of %s are contiguous" % name)
    # the stride of a dimension of one says nothing
    _need(M == 0 or (all(n == 1 or a == b for n, a, b in zip(k.shape, k.stride(), v.stride())) and (D == 1 or k.stride(2) == 1)),
          "k and v have the same strides and contiguous head rows")
    for t, name in ((begin, "begin"), (mem_begin, "mem_begin"), (mem_len, "mem_len")):
        _is(t, name, torch.int32, 1), _dense(t, name)
    _need(begin.shape[0] >= 1, "begin is [requests + 1]")
    n_req = begin.shape[0] - 1
    _need(mem_begin.shape[0] == n_req and mem_len.shape[0] == n_req, "mem_begin and mem_len have one for each request")
    if keep is not None:
        _is(keep, "keep", torch.uint8, 1), _dense(keep, "keep")
        _need(keep.shape[0] == M, "keep is [states]")
    d = wt.CrossDesc(q=_ptr(q), out=_ptr(out), begin=_ptr(begin), k=_ptr(k), v=_ptr(v), mem_begin=_ptr(mem_begin),
                     mem_len=_ptr(mem_len), keep=_ptr(keep), q_stride=q.stride(0) if N > 1 else H * D,
                     out_stride=out.stride(0) if N > 1 else H * D, mem_stride=k.stride(0) if M > 1 else Hkv * D,
                     mem_head=k.stride(1) if Hkv > 1 else D, n_mem=M, dtype=_TYPES[q.dtype], n_req=n_req, n_tokens=N,
                     max_new=max_new, max_mem=max_mem, heads=H, kv_heads=Hkv, head_dim=D,
                     scale=D ** -0.5 if scale is None else scale)
    d.tensors = (q, out, begin, k, v, mem_begin, mem_len, keep)
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


def log_probabilities(logits, *, given=None, given_lp=None, entropy=None, top=None, top_lp=None,
                      temperature=None) -> wt.LogprobsDesc:
    """Log probabilities of given tokens, entropy and the likeliest tokens of each row (see wt_logprobs).

    logits fp32 [rows, vocab]; given int32 [rows, n] (negative: none) with given_lp fp32 [rows, n]; entropy
    fp32 [rows]; top int32 [rows, up to 32] with top_lp fp32; temperature fp32 [rows] (None: 1).  What is
    None is not made."""
    _is(logits, "logits", torch.float32, 2)
    rows, V = logits.shape
    _need((given is None) == (given_lp is None), "given and given_lp come together")
    _need((top is None) == (top_lp is None), "top and top_lp come together")
    d = wt.LogprobsDesc(logits=_ptr(logits), ldl=_rows(logits, "logits"), rows=rows, vocab=V)
    if given is not None:
        _is(given, "given", torch.int32, 2), _is(given_lp, "given_lp", torch.float32, 2), _dense(given_lp, "given_lp")
        _need(given.shape[0] == rows and given_lp.shape == given.shape, "given and given_lp are [%d, tokens]" % rows)
        d.given, d.given_lp, d.n_given, d.given_stride = _ptr(given), _ptr(given_lp), given.shape[1], _rows(given, "given")
    if top is not None:
        _is(top, "top", torch.int32, 2), _is(top_lp, "top_lp", torch.float32, 2), _dense(top, "top"), _dense(top_lp, "top_lp")
        _need(top.shape[0] == rows and top_lp.shape == top.shape and top.shape[1] <= wt.WT_LOGPROBS_MAX_TOP,
              "top and top_lp are [%d, up to %d]" % (rows, wt.WT_LOGPROBS_MAX_TOP))
        d.top, d.top_lp, d.n_top = _ptr(top), _ptr(top_lp), top.shape[1]
    for t, name in ((entropy, "entropy"), (temperature, "temperature")):
        if t is not None:
            _is(t, name, torch.float32, 1), _dense(t, name)
            _need(t.shape[0] == rows, "%s is [rows]" % name)
    d.entropy, d.temp = _ptr(entropy), _ptr(temperature)
    d.tensors = (logits, given, given_lp, entropy, top, top_lp, temperature)
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
