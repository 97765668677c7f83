"""Plain 64-bit implementations of a serving step's operators, for the tests.  They work element by
element from the definitions and share nothing with the library."""
import torch

NAN, INF = float("nan"), float("inf")


def adapt(x, slot, A, B, scale, rank, base):
    """(y, sum |B| |v|, sum |B| sum |A| |x|), each [T, M] in float64 on the CPU."""
    x, A, B, base = (t.double().cpu() for t in (x, A, B, base))
    y, s1, s2 = base.clone(), torch.zeros_like(base), torch.zeros_like(base)
    for t in range(x.shape[0]):
        s = int(slot[t])
        if not 0 <= s < A.shape[0]:
            continue
        r = A.shape[1] if rank is None else min(max(int(rank[s]), 0), A.shape[1])
        c = 1.0 if scale is None else float(scale[s])
        v = A[s, :r] @ x[t]
        y[t] += c * (B[s, :, :r] @ v)
        s1[t] = abs(c) * (B[s, :, :r].abs() @ v.abs())
        s2[t] = abs(c) * (B[s, :, :r].abs() @ (A[s, :r].abs() @ x[t].abs()))
    return y, s1, s2


def attend(q, begin, prefix_k, prefix_v, k_pages, v_pages, table, lens, scale):
    """(out, sum p |v|, the keys' largest sum |q| |k|), float64 on the CPU; rows no request holds stay NaN."""
    q = q.double().cpu()
    N, H, D = q.shape
    pk = None if prefix_k is None else prefix_k.double().cpu()
    pv = None if prefix_v is None else prefix_v.double().cpu()
    Hkv = pk.shape[1] if pk is not None else k_pages.shape[2] if k_pages is not None else H
    page = k_pages.shape[1] if k_pages is not None else 1
    out = torch.full((N, H, D), NAN, dtype=torch.float64)
    mag, qk = torch.zeros_like(out), torch.zeros(N, H, 1, dtype=torch.float64)
    for b in range(len(begin) - 1):
        t0, t1 = int(begin[b]), int(begin[b + 1])
        n = int(lens[b]) if lens is not None else 0
        rows = [(int(table[b][j // page]), j % page) for j in range(n)]
        ok = (lambda a: a.double().cpu())
        ko = [ok(k_pages[p, r]) for p, r in rows]
        vo = [ok(v_pages[p, r]) for p, r in rows]
        for t in range(t0, t1):
            sees = n - (t1 - t0) + 1 + (t - t0)
            k = ([pk] if pk is not None else []) + ([torch.stack(ko[:sees])] if sees > 0 and n else [])
            v = ([pv] if pv is not None else []) + ([torch.stack(vo[:sees])] if sees > 0 and n else [])
            if not k or sum(len(a) for a in k) == 0:
                out[t] = 0
                continue
            k, v = torch.cat(k), torch.cat(v)
            for h in range(H):
                g = h * Hkv // H
                s = scale * (k[:, g] @ q[t, h])
                p = torch.softmax(s, dim=0)
                out[t, h] = p @ v[:, g]
                mag[t, h] = p @ v[:, g].abs()
                qk[t, h] = abs(scale) * float((k[:, g].abs() @ q[t, h].abs()).max())
    return out, mag, qk


def verify(p, q, drafted, begin, u, u_draw, max_draft):
    """(accepted, tokens) in exact integer arithmetic."""
    import numpy as np
    p = p.cpu().numpy()
    q = None if q is None else q.cpu().numpy()
    u, u_draw, drafted, begin = u.tolist(), u_draw.tolist(), drafted.tolist(), begin.tolist()
    acc, toks = [], []

    def weight(x):
        return int(min(float(x), 1.0) * 2.0 ** 40) if x > 0 else 0  # a float times 2^40 is exact

    for b in range(len(begin) - 1):
        n0, n = int(begin[b]), int(begin[b + 1]) - int(begin[b])
        i = 0
        while i < n:
            d = int(drafted[n0 + i])
            if not 0 <= d < p.shape[1]:
                break
            qd = np.float32(1) if q is None else q[n0 + i, d]
            if not np.float32(u[n0 + i]) * qd < p[n0 + b + i, d]:
                break
            i += 1
        row = p[n0 + b + i]
        w = row
        if i < n:
            if q is not None:
                w = row - q[n0 + i]
            else:
                w = row.copy()
                if 0 <= int(drafted[n0 + i]) < p.shape[1]:
                    w[int(drafted[n0 + i])] = 0
        ws = [weight(x) for x in w]
        if sum(ws) == 0:
            ws = [weight(x) for x in row]
        S, tok = sum(ws), -1
        if S:
            limit = (int(float(u_draw[b]) * 2 ** 24) * S) >> 24
            run = 0
            for v, x in enumerate(ws):
                run += x
                if run > limit:
                    tok = v
                    break
        acc.append(i)
        toks.append([int(drafted[n0 + k]) for k in range(i)] + [tok] + [-1] * (max_draft - i))
    return acc, toks
