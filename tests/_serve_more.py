"""Plain 64-bit implementations of placing, attention to memories and log probabilities, for the tests.
They work from the definitions and share nothing with the library."""
import math

import torch

INF = float("inf")


def place_head(x, w, eps, freq, pos, near):
    """(y, magnitude) of heads x [heads, D] of one token; pos [pairs] the position of each pair."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(dim=1, keepdim=True) + eps) * w.double()
    y, mag = x.clone(), x.abs().clone()
    n = len(freq)
    for j in range(n):
        a = math.remainder(float(pos[j]) * freq[j], 2 * math.pi) if abs(pos[j]) < 2 ** 20 else angle(pos[j], freq[j])
        c, s = math.cos(a), math.sin(a)
        i0, i1 = (2 * j, 2 * j + 1) if near else (j, j + n)
        y[:, i0], y[:, i1] = x[:, i0] * c - x[:, i1] * s, x[:, i1] * c + x[:, i0] * s
        mag[:, i0] = mag[:, i1] = x[:, i0].abs() + x[:, i1].abs()
    return y, mag


def angle(pos, f):
    """pos * f modulo a turn, in exact fractions."""
    from fractions import Fraction
    turn = 2 * Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)
    a = Fraction(int(pos)) * Fraction(f)
    return float(a - round(a / turn) * turn)


def place(q, k, v, begin, lens, table, page, q_norm, k_norm, eps, freq, axis, pos, first, near):
    """({token: (y, mag)} of the queries, {(page, row): ((k, mag), (v, mag))})."""
    qs, rows = {}, {}
    cpu = lambda t: None if t is None else t.cpu()  # noqa: E731
    q, k, v, q_norm, k_norm = map(cpu, (q, k, v, q_norm, k_norm))
    begin, lens, table = begin.tolist(), lens.tolist(), table.tolist()
    for b in range(len(begin) - 1):
        n = begin[b + 1] - begin[b]
        for i in range(n):
            t, at = begin[b] + i, lens[b] - n + i
            p = [first + at] * len(freq) if pos is None else [int(pos[t, axis[j]]) for j in range(len(freq))]
            if q is not None:
                qs[t] = place_head(q[t], q_norm, eps, freq, p, near)
            if at >= 0:
                where = (table[b][at // page], at % page)
                rows[where] = (None if k is None else place_head(k[t], k_norm, eps, freq, p, near),
                               None if v is None else place_head(v[t], None, eps, [], [], near))
    return qs, rows


def logprobs(logits, temp):
    """Of one row (1-D): (log p, entropy, mean |x|, mean x^2) with x = (l - m) / t, in float64."""
    l = logits.double().cpu()
    m = l.max()
    if m == -INF:
        return torch.full_like(l, -INF), 0.0, 0.0, 0.0
    if temp <= 0:
        lp = torch.full_like(l, -INF)
        lp[int((l == m).nonzero()[0])] = 0.0
        return lp, 0.0, 0.0, 0.0
    x = (l - m) / temp
    e = torch.exp(x)
    e[int((l == m).nonzero()[0])] = 0.0  # the largest one's 1 apart: a sharp row's sum is near it
    lp = x - torch.log1p(e.sum())
    p, some = torch.exp(lp), x > -INF
    return lp, float(-(p[some] * lp[some]).sum()), float((p[some] * x[some].abs()).sum()), float((p[some] * x[some] ** 2).sum())


def top(logits, n):
    """The n largest logits' tokens, equal ones in order; no NaN, no -infinity."""
    l = logits.tolist()
    order = sorted((v for v in range(len(l)) if l[v] == l[v] and l[v] > -INF), key=lambda v: (-l[v], v))[:n]
    return order + [-1] * (n - len(order))


def cross(q, begin, k, v, mem_begin, mem_len, keep, scale):
    """(out, sum p |v|, the states' largest sum |q| |k|), float64 on the CPU; rows no request holds stay NaN."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    N, H, D = q.shape
    G = H // k.shape[1]
    out = torch.full((N, H, D), float("nan"), dtype=torch.float64)
    mag, qk = torch.zeros_like(out), torch.zeros(N, H, 1, dtype=torch.float64)
    begin, mem_begin, mem_len = begin.tolist(), mem_begin.tolist(), mem_len.tolist()
    for b in range(len(mem_len)):
        t = slice(begin[b], begin[b + 1])
        rows = torch.arange(mem_begin[b], mem_begin[b] + mem_len[b])
        if keep is not None:
            rows = rows[keep.cpu()[rows] != 0]
        if len(rows) == 0:
            out[t] = 0
            continue
        for h in range(H):
            kk, vv = k[rows, h // G], v[rows, h // G]
            s = scale * (q[t, h] @ kk.t())
            top = s.amax(dim=1, keepdim=True)
            e = torch.exp(s - torch.where(top == -INF, torch.zeros_like(top), top))
            p = e / torch.where(top == -INF, torch.ones_like(top), e.sum(dim=1, keepdim=True))
            # a weight of 0 does not hide a value that is not finite
            out[t, h] = p @ vv
            mag[t, h] = p @ vv.abs()
            qk[t, h, 0] = abs(scale) * (q[t, h].abs() @ kk.abs().t()).amax(dim=1)
    return out, mag, qk
