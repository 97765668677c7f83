"""One step of many requests over one set of weights, as cases for timing its operators.

A case is a dict of plain values.  Its `op` names the operator:

  op "adapt"    Handle.adapt: y = base + scale B (A x), each token with its request's low-rank
                adapter, beside the fp32 outputs of a shared projection.  `outs` are the rows M of
                the projections that share x, joined by "+".
  op "attend"   Handle.attend: attention of every request's new tokens over a prefix that all
                share and over the request's own paged cache.
  op "probs"    Handle.probs: fp32 logits to probabilities, a temperature for each row.
  op "verify"   Handle.verify: how many drafted tokens stay, and the token drawn after them, from
                given random numbers.

Structure (lengths, ranks, slots) comes from the case's `pick`, values from the seed.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one token through one square projection of the large decoder: a call's fixed cost
        dict(name="adapt_one_token", op="adapt", dtype="bf16", T=1, reqs=1, K=4096, outs="4096", S=4, R=16, mixed=False, pick=1),
        # a decode step of 48 requests through q, k, v of the large decoder, adapters of mixed ranks
        dict(name="adapt_decode_qkv", op="adapt", dtype="bf16", T=48, reqs=48, K=4096, outs="4096+1024+1024", S=32, R=32, mixed=True, pick=2),
        # a few prompts at once through gate and up of the mid decoder, tokens in runs
        dict(name="adapt_prompts_ffn", op="adapt", dtype="f16", T=4001, reqs=9, K=2560, outs="6912+6912", S=6, R=64, mixed=True, pick=3),
        # one request, one token, a short prefix: latency
        dict(name="attend_one_token", op="attend", dtype="bf16", B=1, new=1, H=32, Hkv=8, D=128, P=500, own=37, page=16, fused=True, pick=4),
        # a decode step of 24 requests behind a system prompt
        dict(name="attend_decode", op="attend", dtype="bf16", B=24, new=1, H=32, Hkv=8, D=128, P=6000, own=900, page=16, fused=True, pick=5),
        # a head for every query, 80 wide (2560 / 32), and pages that end inside tiles
        dict(name="attend_wide_heads", op="attend", dtype="f16", B=7, new=3, H=32, Hkv=32, D=80, P=1021, own=333, page=24, fused=False, pick=6),
        # drafts of up to 4 tokens of 64 requests behind a long document
        dict(name="attend_drafts", op="attend", dtype="bf16", B=64, new=4, H=32, Hkv=8, D=128, P=32768, own=1024, page=64, fused=True, pick=7),
        # the logits of two tokens, one of them drawn greedily
        dict(name="probs_two_rows", op="probs", rows=2, V=32000, greedy=0.5, masked=0.0, pick=8),
        # the logits of 64 requests' drafts over the large decoder's vocabulary, many masked
        dict(name="probs_drafts", op="probs", rows=257, V=128256, greedy=0.1, masked=0.3, pick=9),
        # four drafted tokens of one request
        dict(name="verify_one", op="verify", B=1, new=4, V=32000, certain=False, sharp=3.0, pick=10),
        # 64 requests of up to 4 drafted tokens over the large decoder's vocabulary
        dict(name="verify_batch", op="verify", B=64, new=4, V=128256, certain=False, sharp=2.5, pick=11),
        # drafts copied from the prompt: the draft is certain; an odd vocabulary
        dict(name="verify_copied", op="verify", B=16, new=10, V=50021, certain=True, sharp=6.0, pick=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("adapt", "adapt", "attend", "attend", "attend", "probs", "verify", "verify"))
    pick = rng.randint(0, 9999)
    if op == "adapt":
        d, kv, ffn = rng.choice(((4096, 1024, 14336), (2560, 2560, 6912), (1024, 256, 2731)))
        K, outs = rng.choice(((d, [d, kv, kv]), (d, [d]), (d, [ffn, ffn]), (ffn, [d])))
        T = _log(rng, 1, 4096)
        T = max(1, min(T, 55_000_000 // (sum(outs) + K)))
        c = dict(op=op, dtype=rng.choice(("bf16", "f16")), T=T, reqs=rng.choice((T, max(1, T // 7), 1)), K=K,
                 outs="+".join(map(str, outs)), S=_log(rng, 1, 48), R=rng.choice((4, 8, 16, 16, 32, 33, 64)),
                 mixed=rng.random() < 0.5, pick=pick)
        while c["T"] * c["R"] * c["S"] > 4096 * 64 * 8:  # the plain form's v
            c["S"] = max(1, c["S"] // 2)
            c["T"] = c["T"] if c["S"] > 1 else c["T"] // 2
        c["reqs"] = min(c["reqs"], c["T"])
        return c
    if op == "attend":
        H, Hkv, D = rng.choice(((32, 8, 128), (32, 8, 128), (32, 32, 80), (20, 20, 128), (16, 4, 64), (24, 8, 96), (16, 1, 128)))
        c = dict(op=op, dtype=rng.choice(("bf16", "f16")), B=_log(rng, 1, 64), new=rng.choice((1, 1, 2, 4, 8)), H=H, Hkv=Hkv, D=D,
                 P=rng.choice((0, 1)) if rng.random() < 0.1 else _log(rng, 30, 32768), own=_log(rng, 9, 2048),
                 page=rng.choice((1, 16, 16, 24, 64, 128)), fused=rng.random() < 0.5, pick=pick)
        while c["B"] * c["new"] * H * c["P"] > 64 * 2 * 32 * 32768 or c["B"] * c["own"] * Hkv * D > 64 * 1024 * 8 * 128:
            if c["B"] > 1:
                c["B"] //= 2
            else:
                c["P"] //= 2
        return c
    if op == "probs":
        V = _log(rng, 300, 200_000)
        return dict(op=op, rows=max(1, min(_log(rng, 1, 400), 32_000_000 // V)), V=V, greedy=rng.choice((0.0, 0.1, 1.0)),
                    masked=rng.choice((0.0, 0.5, 0.99)), pick=pick)
    V = _log(rng, 300, 200_000)
    new = rng.randint(1, 12)
    return dict(op=op, B=max(1, min(_log(rng, 1, 64), 40_000_000 // (V * new))), new=new, V=V, certain=rng.random() < 0.3,
                sharp=rng.choice((1.0, 2.5, 6.0)), pick=pick)


# ------------------------------------------------------------------------------ structure, from the case alone

def _outs(case):
    return [int(m) for m in case["outs"].split("+")]


def _slots(case):
    """(slot of each token, rank of each slot, scale of each slot); one request in nine has no adapter."""
    r = random.Random(case["pick"])
    of = [r.randrange(case["S"]) if r.random() < 8 / 9 or case["reqs"] == 1 else -1 for _ in range(case["reqs"])]
    slot = [of[t * case["reqs"] // case["T"]] for t in range(case["T"])]
    rank = [r.randint(1, case["R"]) if case["mixed"] else case["R"] for _ in range(case["S"])]
    return slot, rank, [16.0 / n for n in rank]


def _requests(case):
    """(new tokens of each request, own keys of each request, its new tokens' among them)."""
    r = random.Random(case["pick"])
    new = [r.randint(max(1, case["new"] // 2), case["new"]) for _ in range(case["B"])]
    return new, [r.randint(n, max(n, case["own"])) for n in new]


def _drafts(case):
    """Drafted tokens of each request: none for some."""
    r = random.Random(case["pick"])
    return [r.randint(0 if case["B"] > 1 else 1, case["new"]) for _ in range(case["B"])]


def _begin(counts):
    b = [0]
    for n in counts:
        b.append(b[-1] + n)
    return b


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------ inputs

class _State:
    pass


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(int(seed))
    s = _State()
    s.case = case

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    def rand(*shape):
        return torch.rand(shape, device="cuda", generator=g)

    if case["op"] == "adapt":
        dt = DTYPES[case["dtype"]]
        T, K, S, R = case["T"], case["K"], case["S"], case["R"]
        slot, rank, scale = _slots(case)
        s.slot, s.rank, s.scale = _ints(slot), _ints(rank), torch.tensor(scale, device="cuda")
        s.x = normal(T, K, dtype=dt)
        s.A = [normal(S, R, K, std=K ** -0.5, dtype=dt) for _ in _outs(case)]
        s.B = [normal(S, M, R, std=0.02, dtype=dt) for M in _outs(case)]
        s.base = [normal(T, M) for M in _outs(case)]
        s.y = [torch.empty(T, M, device="cuda") for M in _outs(case)]
    elif case["op"] == "attend":
        dt = DTYPES[case["dtype"]]
        B, H, Hkv, D, P, page = (case[k] for k in ("B", "H", "Hkv", "D", "P", "page"))
        new, lens = _requests(case)
        N = sum(new)
        s.begin, s.lens, s.max_new, s.max_len = _ints(_begin(new)), _ints(lens), max(new), max(lens)
        # queries as a fused q, k, v projection leaves them, or on their own
        s.q = normal(N, H + 2 * Hkv if case["fused"] else H, D, std=1.5, dtype=dt)[:, :H]
        s.pk, s.pv = normal(P, Hkv, D, dtype=dt), normal(P, Hkv, D, dtype=dt)
        pages = [-(-n // page) for n in lens]
        most, total = max(pages), sum(pages) + 3
        order = list(range(total))
        random.Random(case["pick"] + 1).shuffle(order)
        first = _begin(pages)
        s.table = _ints([[order[first[b] + j] if j < pages[b] else -1 for j in range(most)] for b in range(B)])
        s.k, s.v = normal(total, page, Hkv, D, dtype=dt), normal(total, page, Hkv, D, dtype=dt)
        # a pool's pages hold anything past a request's last key
        at = torch.arange(most * page, device="cuda").view(1, most, page)
        past = torch.zeros(total, page, dtype=torch.bool, device="cuda")
        past[s.table.clamp(min=0).long().view(-1)] = (at >= s.lens.view(-1, 1, 1)).view(-1, page) & (s.table.view(-1, 1) >= 0)
        s.k[past], s.v[past] = float("nan"), float("inf")
        s.scale = D ** -0.5
        s.out = torch.empty(N, H, D, dtype=dt, device="cuda")
    elif case["op"] == "probs":
        rows, V = case["rows"], case["V"]
        s.logits = normal(rows, V, std=3.0)
        s.logits[rand(rows, V) < case["masked"]] = -float("inf")
        s.temp = torch.where(rand(rows) < case["greedy"], torch.zeros(rows, device="cuda"), 0.3 + rand(rows))
        s.p = torch.empty(rows, V, device="cuda")
    else:
        V, drafts = case["V"], _drafts(case)
        B, n = case["B"], sum(drafts)
        s.max_draft = case["new"]
        s.begin = _ints(_begin(drafts))
        of = torch.repeat_interleave(torch.arange(B, device="cuda"), s.begin.diff().long())
        row = torch.arange(n, device="cuda") + of  # a request has one row more than drafted tokens
        logits = normal(n + B, V, std=case["sharp"])
        s.p = torch.softmax(logits, dim=1)
        if case["certain"]:
            s.q = None
            s.drafted = torch.where(rand(n) < 0.7, logits[row].argmax(dim=1), (rand(n) * V).long().clamp(max=V - 1)).int()
        else:
            s.q = torch.softmax(logits[row] + normal(n, V, std=0.5), dim=1)
            c = torch.cumsum(s.q, dim=1, dtype=torch.float64)
            s.drafted = (c < rand(n, 1).double() * c[:, -1:]).sum(dim=1).clamp(max=V - 1).int()
        s.u, s.u_draw = rand(n), rand(B)
        s.accepted = torch.empty(B, dtype=torch.int32, device="cuda")
        s.tokens = torch.empty(B, s.max_draft + 1, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handle and the descriptors that a program keeps from step to step
        from paper_2608_12114_gb300 import serving, wt
        s.h = wt.Handle([])
        if case["op"] == "adapt":
            s.descs = [serving.adapters(s.x, s.y[i], s.slot, s.A[i], s.B[i], s.scale, rank=s.rank, base=s.base[i])
                       for i in range(len(s.A))]
        elif case["op"] == "attend":
            s.desc = serving.attention(s.q, s.out, s.begin, s.k, s.v, s.table, s.lens, max_new=s.max_new, max_len=s.max_len,
                                       prefix_k=s.pk, prefix_v=s.pv, scale=s.scale)
        elif case["op"] == "probs":
            s.desc = serving.probabilities(s.logits, s.p, temperature=s.temp)
        else:
            s.desc = serving.verification(s.p, s.drafted, s.begin, s.u, s.u_draw, s.accepted, s.tokens, q=s.q)
    return s


# ------------------------------------------------------------------------------ the operators

def run(s):
    op = s.case["op"]
    if not own:
        return {"adapt": _adapt, "attend": _attend, "probs": _probs, "verify": _verify}[op](s)
    stream = torch.cuda.current_stream().cuda_stream
    if op == "adapt":
        s.h.adapt(s.descs, stream)
        return s.y
    if op == "attend":
        s.h.attend(s.desc, stream)
        return s.out
    if op == "probs":
        s.h.probs(s.desc, stream)
        return s.p
    s.h.verify(s.desc, stream)
    return s.accepted, s.tokens


def _adapt(s):
    S, R, K = s.A[0].shape
    x = s.x.float()
    mine = (s.slot.view(-1, 1, 1) == torch.arange(S, device="cuda").view(1, S, 1)) & \
           (torch.arange(R, device="cuda") < s.rank.view(S, 1))  # [T, S, R]
    coef = torch.where(mine, s.scale.view(1, S, 1), torch.zeros((), device="cuda")).view(-1, S * R)
    y = []
    for A, B, base in zip(s.A, s.B, s.base):  # the projections that share x
        v = torch.matmul(x, A.float().view(S * R, K).t()) * coef
        y.append(base + torch.matmul(v, B.float().transpose(1, 2).reshape(S * R, -1)))
    return y


def _attend(s):
    N, H, D = s.q.shape
    P, Hkv, _ = s.pk.shape
    B, L, G, page = len(s.lens), s.max_len, H // Hkv, s.k.shape[1]
    begin, lens = s.begin.long(), s.lens.long()
    t = torch.arange(N, device="cuda")
    b = torch.searchsorted(begin, t, right=True) - 1
    i = t - begin[b]
    q = s.q.float() * s.scale
    qp = torch.zeros(B, s.max_new, H, D, device="cuda")
    qp[b, i] = q
    qp = qp.view(B, s.max_new, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, s.max_new * G, D)
    j = torch.arange(L, device="cuda")
    at = s.table.clamp(min=0).long()[:, j // page] * page + j % page  # [B, L]
    there = (j < lens.view(B, 1)).view(B, L, 1, 1)
    zero = torch.zeros((), device="cuda")
    k = torch.where(there, s.k.view(-1, Hkv, D)[at].float(), zero).permute(0, 2, 1, 3)  # [B, Hkv, L, D]
    v = torch.where(there, s.v.view(-1, Hkv, D)[at].float(), zero).permute(0, 2, 1, 3)
    sees = (lens - begin.diff()).view(B, 1) + 1 + torch.arange(s.max_new, device="cuda")  # own keys each token sees
    sees = sees.clamp(max=L).repeat_interleave(G, dim=1).view(B, 1, -1, 1)
    so = torch.where(j < sees, torch.matmul(qp, k.transpose(2, 3)), torch.full((), -float("inf"), device="cuda"))
    qt = q.view(N, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, N * G, D)
    pad = lambda x: torch.zeros(B, s.max_new, Hkv, G, x.shape[-1], device="cuda").index_put_(  # noqa: E731
        (b, i), x.view(Hkv, N, G, -1).permute(1, 0, 2, 3)).permute(0, 2, 1, 3, 4).reshape(B, Hkv, s.max_new * G, -1)
    flat = lambda x: x.view(B, Hkv, s.max_new, G, -1).permute(0, 2, 1, 3, 4)[b, i]  # noqa: E731  [N, Hkv, G, .]
    m = flat(so.amax(dim=3, keepdim=True)).permute(1, 0, 2, 3).reshape(Hkv, N * G, 1)
    if P:
        sp = torch.matmul(qt, s.pk.float().permute(1, 2, 0))  # [Hkv, N G, P]
        m = torch.maximum(m, sp.amax(dim=2, keepdim=True))
    m = torch.where(m > -float("inf"), m, zero)
    eo = torch.exp(so - pad(m))
    num, den = flat(torch.matmul(eo, v)), flat(eo.sum(dim=3, keepdim=True))
    if P:
        ep = torch.exp(sp - m)
        num = num + torch.matmul(ep, s.pv.float().permute(1, 0, 2)).view(Hkv, N, G, D).permute(1, 0, 2, 3)
        den = den + ep.sum(dim=2).view(Hkv, N, G, 1).permute(1, 0, 2, 3)
    o = torch.where(den > 0, num / den, zero)
    return o.reshape(N, H, D).to(s.q.dtype)


def _probs(s):
    m = s.logits.amax(dim=1, keepdim=True)
    some = m > -float("inf")
    first = s.logits.argmax(dim=1, keepdim=True) == torch.arange(s.logits.shape[1], device="cuda")
    t = s.temp.view(-1, 1)
    e = torch.exp((s.logits - torch.where(some, m, torch.zeros_like(m))) / torch.where(t > 0, t, torch.ones_like(t)))
    e = torch.where(t > 0, e, first.float())
    return torch.where(some, e / e.sum(dim=1, keepdim=True), torch.zeros_like(e))


def _verify(s):
    V, B, n = s.p.shape[1], len(s.u_draw), len(s.drafted)
    begin = s.begin.long()
    drafts = begin.diff()
    of = torch.repeat_interleave(torch.arange(B, device="cuda"), drafts, output_size=n)
    d = s.drafted.long().view(-1, 1)
    pd = s.p[torch.arange(n, device="cuda") + of].gather(1, d).view(-1) if n else s.u
    qd = torch.ones_like(pd) if s.q is None else s.q.gather(1, d).view(-1)
    i = torch.arange(s.max_draft, device="cuda")
    at = (begin[:-1].view(B, 1) + i).clamp(max=max(n - 1, 0))
    stays = (s.u * qd < pd)[at] & (i < drafts.view(B, 1)) if n else torch.zeros(B, s.max_draft, dtype=torch.bool, device="cuda")
    accepted = torch.cumprod(stays.long(), dim=1).sum(dim=1)
    refused = accepted < drafts
    p = s.p[begin[:-1] + torch.arange(B, device="cuda") + accepted]
    w = p
    if n:
        last = (begin[:-1] + accepted).clamp(max=n - 1)
        one = (torch.arange(V, device="cuda") == d[last]).float() if s.q is None else s.q[last]
        w = torch.where(refused.view(B, 1), torch.clamp(p - one, min=0.0), p)
    whole = lambda x: (torch.clamp(x, max=1.0) * 2.0 ** 40).long()  # noqa: E731
    w = whole(w)
    w = torch.where((w.sum(dim=1) > 0).view(B, 1), w, whole(p))
    run_sum = torch.cumsum(w, dim=1)
    S = run_sum[:, -1]
    u = (s.u_draw * 2.0 ** 24).long()
    limit = u * (S >> 24) + ((u * (S & ((1 << 24) - 1))) >> 24)
    token = torch.where(S > 0, (run_sum <= limit.view(B, 1)).sum(dim=1), torch.full_like(S, -1))
    i = torch.arange(s.max_draft + 1, device="cuda")
    tokens = torch.full((B, s.max_draft + 1), -1, dtype=torch.int64, device="cuda")
    if n:
        at = (begin[:-1].view(B, 1) + i).clamp(max=n - 1)
        tokens = torch.where(i < accepted.view(B, 1), d.view(-1)[at], tokens)
    tokens = torch.where(i == accepted.view(B, 1), token.view(B, 1), tokens)
    return accepted.int(), tokens.int()


# ------------------------------------------------------------------------------ what is asked of them

def work(case):
    if case["op"] == "adapt":
        slot, rank, _ = _slots(case)
        outs, used = _outs(case), set(slot) - {-1}
        r = sum(rank[i] for i in used)
        b = sum(2 * r * (case["K"] + M) + 8 * case["T"] * M for M in outs) + 2 * case["T"] * case["K"] + 4 * case["T"]
        return {"bytes": b, "flops": sum(2 * rank[i] * (case["K"] + M) for M in outs for i in slot if i >= 0)}
    if case["op"] == "attend":
        new, lens = _requests(case)
        H, Hkv, D, P = (case[k] for k in ("H", "Hkv", "D", "P"))
        sees = sum(n * (P + m - n) + n * (n + 1) // 2 for n, m in zip(new, lens))
        return {"bytes": 4 * Hkv * D * (P + sum(lens)) + 4 * sum(new) * H * D, "flops": 4 * H * D * sees}
    if case["op"] == "probs":
        return {"bytes": 8 * case["rows"] * case["V"], "flops": 0}
    # the deciding rows: of p for each request, of q for each that refuses a token (about all that
    # have drafts; the point of a certain draft is no row)
    drafts = _drafts(case)
    return {"bytes": 4 * case["V"] * (len(drafts) + (0 if case["certain"] else sum(n > 0 for n in drafts))), "flops": 0}


def exact(case, seed):
    if case["op"] == "verify":
        return None
    s = _inputs(case, seed)
    if case["op"] == "probs":
        l = s.logits.double()
        out = torch.empty_like(l)
        for r in range(case["rows"]):
            t = float(s.temp[r])
            if l[r].max() == -float("inf"):
                out[r] = 0
            elif t > 0:
                out[r] = torch.softmax((l[r] - l[r].max()) / t, dim=0)
            else:
                out[r] = 0
                out[r, int((l[r] == l[r].max()).nonzero()[0])] = 1
        return out
    if case["op"] == "adapt":
        slot, rank, scale = _slots(case)
        slot = torch.tensor(slot, device="cuda")
        y = []
        for A, B, base in zip(s.A, s.B, s.base):
            o = base.double()
            for i in range(case["S"]):
                t = (slot == i).nonzero().view(-1)
                if len(t):
                    v = torch.mm(s.x[t].double(), A[i, :rank[i]].double().t())
                    o[t] += float(s.scale[i]) * torch.mm(v, B[i, :, :rank[i]].double().t())
            y.append(o)
        return y
    new, lens = _requests(case)
    H, Hkv, D, page = (case[k] for k in ("H", "Hkv", "D", "page"))
    G, first = H // Hkv, _begin(new)
    table = s.table.tolist()
    out = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
    pk, pv = s.pk.double(), s.pv.double()
    for b, (n, m) in enumerate(zip(new, lens)):
        at = torch.tensor([table[b][j // page] * page + j % page for j in range(m)], device="cuda")
        k = torch.cat([pk, s.k.view(-1, Hkv, D)[at].double()])
        v = torch.cat([pv, s.v.view(-1, Hkv, D)[at].double()])
        hide = torch.arange(len(k), device="cuda") >= case["P"] + m - n + 1 + torch.arange(n, device="cuda").view(n, 1)
        for h in range(Hkv):
            q = s.q[first[b]:first[b] + n, h * G:(h + 1) * G].double()
            a = (torch.einsum("ngd,kd->ngk", q, k[:, h]) * D ** -0.5).masked_fill(hide.view(n, 1, -1), -float("inf"))
            out[first[b]:first[b] + n, h * G:(h + 1) * G] = torch.einsum("ngk,kd->ngd", torch.softmax(a, dim=2), v[:, h])
    return out
