"""What a step of many requests does around its products and its attention, as cases for timing.

A case is a dict of plain values.  Its `op` names the operator:

  op "place"     Handle.place: the projections' rows to queries and cached keys and values: norms of
                 each head, rotation by position (of one axis or several), cast, and the new keys and
                 values into their requests' pages.
  op "cross"     Handle.cross: attention of every request's tokens to a memory of its own, such as an
                 encoder's states, of any length and with states left out.
  op "logprobs"  Handle.logprobs: log probabilities of given tokens, entropy, and the likeliest
                 tokens of fp32 logits, a temperature for each row.

Structure (lengths, pages, axes) comes from the case's `pick`, values from the seed.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one new token of one request through a layer of the large decoder: a call's fixed cost
        dict(name="place_one_token", op="place", src="f32", dtype="bf16", B=1, new=1, past=700, pad=0, H=32, Hkv=8, D=128, rot=128,
             near=False, axes=1, far=False, norm="none", page=16, pick=1),
        # drafts of up to 4 tokens of 64 requests, a norm for each head of q and k, positions past a million
        dict(name="place_drafts", op="place", src="f32", dtype="bf16", B=64, new=4, past=1024, pad=0, H=32, Hkv=8, D=128, rot=128,
             near=False, axes=1, far=True, norm="bf16", page=64, pick=2),
        # a prompt with images: positions of three axes, rows of a fused projection in 16 bits
        dict(name="place_images", op="place", src="bf16", dtype="bf16", B=3, new=2001, past=0, pad=0, H=20, Hkv=20, D=128, rot=128,
             near=False, axes=3, far=False, norm="bf16", page=16, pick=3),
        # prompts behind earlier turns, half of each head rotated, odd pages, padded rows behind the last
        dict(name="place_prompts", op="place", src="f32", dtype="f16", B=9, new=1500, past=333, pad=61, H=32, Hkv=32, D=80, rot=40,
             near=True, axes=1, far=False, norm="none", page=24, pick=4),
        # one token of one request, an encoder's states: latency
        dict(name="cross_one_token", op="cross", dtype="bf16", B=1, new=1, H=32, Hkv=8, D=128, mem=1500, holes=0.0, fused=False, pick=5),
        # a decode step of 48 requests, a head for every query
        dict(name="cross_decode", op="cross", dtype="bf16", B=48, new=1, H=20, Hkv=20, D=64, mem=1500, holes=0.0, fused=False, pick=6),
        # a few beams or drafts each, heads of 80, keys and values of one projection, states left out
        dict(name="cross_beams", op="cross", dtype="f16", B=13, new=5, H=32, Hkv=32, D=80, mem=777, holes=0.3, fused=True, pick=7),
        # targets of six requests at once, as a prompt or for scoring
        dict(name="cross_targets", op="cross", dtype="bf16", B=6, new=448, H=20, Hkv=20, D=64, mem=1500, holes=0.0, fused=True, pick=8),
        # two long texts against long memories
        dict(name="cross_long", op="cross", dtype="bf16", B=2, new=1024, H=32, Hkv=8, D=128, mem=16384, holes=0.0, fused=False, pick=9),
        # the tokens of two requests and five alternatives
        dict(name="logprobs_two_rows", op="logprobs", rows=2, V=32000, given=1, top=5, greedy=0.0, masked=0.0, pick=10),
        # 64 requests' drafts over the large decoder's vocabulary, many tokens masked, twenty alternatives
        dict(name="logprobs_drafts", op="logprobs", rows=257, V=128256, given=1, top=20, greedy=0.1, masked=0.3, pick=11),
        # a text scored token by token, an odd vocabulary
        dict(name="logprobs_text", op="logprobs", rows=2047, V=50021, given=1, top=0, greedy=0.0, masked=0.0, pick=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 8, 128), (32, 8, 128), (32, 32, 80), (20, 20, 128), (20, 20, 64), (16, 4, 64), (24, 8, 96), (16, 1, 128))


def draw(rng):
    op = rng.choice(("place", "place", "cross", "cross", "cross", "logprobs", "logprobs"))
    pick = rng.randint(0, 9999)
    if op == "place":
        H, Hkv, D = rng.choice(HEADS)
        dt = rng.choice(("bf16", "f16"))
        c = dict(op=op, src=rng.choice(("f32", dt)), dtype=dt, B=_log(rng, 1, 64), new=_log(rng, 1, 2000), past=rng.choice((0, _log(rng, 1, 1500))),
                 pad=rng.choice((0, 0, rng.randint(1, 70))), H=H, Hkv=Hkv, D=D, rot=rng.choice((D, D, D // 16 * 8, 0)), near=rng.random() < 0.3,
                 axes=rng.choice((1, 1, 2, 3)), far=rng.random() < 0.3, norm=rng.choice(("none", "f32", dt)), page=rng.choice((1, 16, 24, 64)), pick=pick)
        while c["B"] * c["new"] * (H + 2 * Hkv) * D > 9 * 1500 * 96 * 80 or c["B"] * (c["new"] + c["past"]) * Hkv * D > 9 * 1833 * 32 * 80:
            if c["B"] > 1:
                c["B"] //= 2
            elif c["past"] > c["new"]:
                c["past"] //= 2
            else:
                c["new"] //= 2
        return c
    if op == "cross":
        H, Hkv, D = rng.choice(HEADS)
        c = dict(op=op, dtype=rng.choice(("bf16", "f16")), B=_log(rng, 1, 64), new=rng.choice((1, 1, 2, _log(rng, 3, 1024))), H=H, Hkv=Hkv, D=D,
                 mem=_log(rng, 1, 16384), holes=rng.choice((0.0, 0.0, 0.0, 0.2, 0.9)), fused=rng.random() < 0.5, pick=pick)
        while c["B"] * c["new"] * c["mem"] * H > 2 * 1024 * 16384 * 16 or c["B"] * c["mem"] * Hkv * D > 64 * 1500 * 20 * 64:
            if c["B"] > 1:
                c["B"] //= 2
            elif c["new"] * 16 > c["mem"]:
                c["new"] //= 2
            else:
                c["mem"] //= 2
        return c
    V = _log(rng, 300, 200_000)
    return dict(op=op, rows=max(1, min(_log(rng, 1, 2000), 33_000_000 // V)), V=V, given=rng.choice((0, 1, 1, 4)),
                top=rng.choice((0, 1, 5, 20, 32)), greedy=rng.choice((0.0, 0.1, 1.0)), masked=rng.choice((0.0, 0.5, 0.999)), pick=pick)


# ------------------------------------------------------------------------------ structure, from the case alone

def _placed(case):
    """(new tokens of each request, its own keys with the new tokens' among them)."""
    r = random.Random(case["pick"])
    new = [r.randint(max(1, case["new"] // 2), case["new"]) for _ in range(case["B"])]
    return new, [n + r.randint(case["past"] // 2, case["past"]) for n in new]


def _axes(case):
    """The axis of each pair: runs of pairs, or each axis in turn."""
    pairs, n = case["rot"] // 2, case["axes"]
    return [j % n if case["pick"] % 2 == 0 else j * n // pairs for j in range(pairs)]


def _memories(case):
    """(tokens of each request, states of its memory); few requests have none."""
    r = random.Random(case["pick"])
    new = [r.randint(max(1, case["new"] // 2), case["new"]) for _ in range(case["B"])]
    return new, [0 if case["B"] > 8 and r.random() < 0.05 else r.randint(case["mem"] // 2 + 1, case["mem"]) for _ in new]


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

    if case["op"] == "place":
        src, dt = DTYPES[case["src"]], DTYPES[case["dtype"]]
        H, Hkv, D, page, rot = (case[k] for k in ("H", "Hkv", "D", "page", "rot"))
        new, lens = _placed(case)
        N = sum(new) + case["pad"]
        s.begin, s.lens, s.max_len = _ints(_begin(new)), _ints(lens), max(lens)
        if src == torch.float32:  # a buffer for each projection
            s.q, s.k, s.v = normal(N, H, D, dtype=src), normal(N, Hkv, D, dtype=src), normal(N, Hkv, D, dtype=src)
        else:  # one for all three
            s.q, s.k, s.v = normal(N, H + 2 * Hkv, D, dtype=src).split((H, Hkv, Hkv), dim=1)
        nt = None if case["norm"] == "none" else DTYPES[case["norm"]]
        s.q_norm, s.k_norm = (None, None) if nt is None else ((1 + normal(D, std=0.1)).to(nt), (1 + normal(D, std=0.1)).to(nt))
        s.eps = 1e-6
        # radians a position, in 64 bits
        s.freq = [500000.0 ** (-2.0 * j / rot) for j in range(rot // 2)] if rot else None
        s.axis = _axes(case) if rot and case["axes"] > 1 else None
        s.first, s.pos = 1_000_000 if case["far"] else 0, None
        if rot and case["axes"] > 1:
            s.pos = (rand(N, case["axes"]) * torch.tensor([4000.0, 90.0, 120.0], device="cuda")[:case["axes"]]).int() + s.first
        pages = [-(-n // page) for n in lens]
        most, total = max(pages), sum(pages) + 3
        order = list(range(total))
        random.Random(case["pick"] + 1).shuffle(order)
        first = _begin(pages)
        s.table = _ints([[order[first[b] + j] if j < pages[b] else -1 for j in range(most)] for b in range(case["B"])])
        s.k_pages, s.v_pages = normal(total, page, Hkv, D, dtype=dt), normal(total, page, Hkv, D, dtype=dt)
        s.q_out = torch.zeros(N, H, D, dtype=dt, device="cuda")
    elif case["op"] == "cross":
        dt = DTYPES[case["dtype"]]
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        new, mem = _memories(case)
        N, M = sum(new), sum(mem)
        s.begin, s.mem_begin, s.mem_len = _ints(_begin(new)), _ints(_begin(mem)[:-1]), _ints(mem)
        s.max_new, s.max_mem = max(new), max(mem)
        s.q = normal(N, H, D, std=1.5, dtype=dt)
        if case["fused"]:
            s.k, s.v = normal(M, 2, Hkv, D, dtype=dt).unbind(dim=1)
        else:
            s.k, s.v = normal(M, Hkv, D, dtype=dt), normal(M, Hkv, D, dtype=dt)
        s.keep = None
        if case["holes"]:
            s.keep = (rand(M) >= case["holes"]).to(torch.uint8)
            gone = s.keep == 0  # what stands there is anything
            s.k[gone], s.v[gone] = float("nan"), float("inf")
        s.scale = D ** -0.5
        s.out = torch.empty(N, H, D, dtype=dt, device="cuda")
    else:
        rows, V = case["rows"], case["V"]
        s.logits = normal(rows, V, std=3.0)
        s.logits[rand(rows, V) < case["masked"]] = -float("inf")
        s.temp = torch.where(rand(rows) < case["greedy"], torch.zeros(rows, device="cuda"), 0.3 + rand(rows))
        s.given = torch.minimum((rand(rows, case["given"]) * V).int(), _ints(V - 1))
        s.given[:, 1:] = torch.where(rand(*s.given[:, 1:].shape) < 0.3, _ints(-1), s.given[:, 1:])  # rows with fewer tokens
        s.given_lp = torch.empty(rows, case["given"], device="cuda")
        s.entropy = torch.empty(rows, device="cuda")
        s.top = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
        s.top_lp = torch.empty(rows, case["top"], device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "place" and s.freq:
        s.freq64 = torch.tensor(s.freq, dtype=torch.float64, device="cuda")
        s.axis_of = torch.tensor(s.axis or [0] * len(s.freq), device="cuda")
    if own:  # the handle and the descriptor that a program keeps from step to step
        from paper_2608_12114_gb300 import serving, wt
        s.h = wt.Handle([])
        if case["op"] == "place":
            s.desc = serving.placement(s.begin, s.k_pages, s.v_pages, s.table, s.lens, q=s.q, q_out=s.q_out, k=s.k, v=s.v, max_len=s.max_len,
                                       q_norm=s.q_norm, k_norm=s.k_norm, eps=s.eps, turns=serving.turns(s.freq) if s.freq else None,
                                       axis=s.axis, pos=s.pos, first_pos=s.first, neighbours=case["near"])
        elif case["op"] == "cross":
            s.desc = serving.cross_attention(s.q, s.out, s.begin, s.k, s.v, s.mem_begin, s.mem_len, max_new=s.max_new, max_mem=s.max_mem,
                                             keep=s.keep, scale=s.scale)
        else:
            s.desc = serving.log_probabilities(s.logits, given=s.given, given_lp=s.given_lp, entropy=s.entropy, top=s.top, top_lp=s.top_lp,
                                               temperature=s.temp)
    return s


# ------------------------------------------------------------------------------ the operators

def run(s):
    op = s.case["op"]
    if not own:
        return {"place": _place, "cross": _cross, "logprobs": _logprobs}[op](s)
    stream = torch.cuda.current_stream().cuda_stream
    if op == "place":
        s.h.place(s.desc, stream)
        return s.q_out, s.k_pages, s.v_pages
    if op == "cross":
        s.h.cross(s.desc, stream)
        return s.out
    s.h.logprobs(s.desc, stream)
    return s.given_lp, s.entropy, s.top, s.top_lp


def _place(s):
    case = s.case
    D, page, rot = case["D"], case["page"], case["rot"]
    n = len(s.q) - case["pad"]
    begin, lens = s.begin.long(), s.lens.long()
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(begin, t, right=True) - 1
    own_at = lens[b] - begin.diff()[b] + t - begin[b]
    if rot:
        pos = (s.first + own_at).view(n, 1) if s.pos is None else s.pos[:n].long()
        a = pos.double()[:, s.axis_of] * s.freq64  # [n, pairs]
        cos, sin = torch.cos(a).float().view(n, 1, -1), torch.sin(a).float().view(n, 1, -1)

    def turned(x, w):
        x = x[:n].float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(dim=2, keepdim=True) + s.eps) * w.float()
        if not rot:
            return x
        if case["near"]:
            x0, x1 = x[..., 0:rot:2], x[..., 1:rot:2]
            r = torch.stack([x0 * cos - x1 * sin, x1 * cos + x0 * sin], dim=-1).flatten(2)
        else:
            x0, x1 = x[..., :rot // 2], x[..., rot // 2:rot]
            r = torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], dim=2)
        return torch.cat([r, x[..., rot:]], dim=2) if rot < D else r

    dt = s.q_out.dtype
    row = s.table.long()[b, own_at // page] * page + own_at % page
    s.q_out[:n] = turned(s.q, s.q_norm).to(dt)
    s.k_pages.view(-1, case["Hkv"], D)[row] = turned(s.k, s.k_norm).to(dt)
    s.v_pages.view(-1, case["Hkv"], D)[row] = s.v[:n].to(dt)
    return s.q_out, s.k_pages, s.v_pages


def _cross(s):
    N, H, D = s.q.shape
    Hkv = s.k.shape[1]
    B, L, G = len(s.mem_len), s.max_mem, H // Hkv
    begin, lens = s.begin.long(), s.mem_len.long()
    t = torch.arange(N, device="cuda")
    b = torch.searchsorted(begin, t, right=True) - 1
    i = t - begin[b]
    qp = torch.zeros(B, s.max_new, H, D, device="cuda")
    qp[b, i] = s.q.float() * s.scale
    qp = qp.view(B, s.max_new, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, s.max_new * G, D)
    j = torch.arange(L, device="cuda")
    there = j < lens.view(B, 1)
    at = torch.where(there, s.mem_begin.long().view(B, 1) + j, torch.zeros_like(j))
    if s.keep is not None:
        there = there & (s.keep[at] != 0)
    zero = torch.zeros((), device="cuda")
    pick = lambda x: torch.where(there.view(B, L, 1, 1), x[at].float(), zero).permute(0, 2, 1, 3)  # noqa: E731  [B, Hkv, L, D]
    sc = torch.matmul(qp, pick(s.k).transpose(2, 3)).masked_fill_(~there.view(B, 1, 1, L), -float("inf"))
    m = sc.amax(dim=3, keepdim=True)
    e = torch.exp(sc.sub_(torch.where(m > -float("inf"), m, zero)))
    den = e.sum(dim=3, keepdim=True)
    o = torch.where(den > 0, torch.matmul(e, pick(s.v)) / den, zero)
    return o.view(B, Hkv, s.max_new, G, D).permute(0, 2, 1, 3, 4)[b, i].reshape(N, H, D).to(s.q.dtype)


def _logprobs(s):
    V = s.logits.shape[1]
    inf = torch.full((), float("inf"), device="cuda")
    zero = torch.zeros((), device="cuda")
    m = s.logits.amax(dim=1, keepdim=True)
    m = torch.where(m > -inf, m, zero)
    t = s.temp.view(-1, 1)
    x = (s.logits - m) / torch.where(t > 0, t, torch.ones_like(t))
    # a temperature of 0: the first of the largest logits is certain
    first = s.logits.argmax(dim=1, keepdim=True) == torch.arange(V, device="cuda")
    x = torch.where(t > 0, x, torch.where(first & (s.logits > -inf), zero, -inf))
    e = torch.exp(x)
    S = e.sum(dim=1, keepdim=True)
    none = S == 0
    log_S = torch.log(torch.where(none, torch.ones_like(S), S))
    H = log_S - torch.where(e > 0, e * x, zero).sum(dim=1, keepdim=True) / torch.where(none, torch.ones_like(S), S)
    given = s.given.long()
    lp = torch.where(given >= 0, x.gather(1, given.clamp(min=0)) - log_S, zero)
    k = s.top.shape[1]
    if k == 0:
        return lp, H.view(-1), s.top, s.top_lp
    v, at = torch.sort(s.logits, dim=1, descending=True, stable=True)  # equal logits in the order of their tokens
    v, at = v[:, :k], at[:, :k]
    return lp, H.view(-1), torch.where(v > -inf, at, torch.full_like(at, -1)).int(), x.gather(1, at) - log_S


# ------------------------------------------------------------------------------ what is asked of them

def work(case):
    if case["op"] == "place":
        new, _ = _placed(case)
        n, h = sum(new), case["H"] + 2 * case["Hkv"]
        return {"bytes": n * h * case["D"] * ((4 if case["src"] == "f32" else 2) + 2), "flops": 0}
    if case["op"] == "cross":
        new, mem = _memories(case)
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        share = 1.0 - case["holes"]
        return {"bytes": int(4 * Hkv * D * sum(mem) * share) + 4 * sum(new) * H * D,
                "flops": int(4 * H * D * sum(n * m for n, m in zip(new, mem)) * share)}
    return {"bytes": 4 * case["rows"] * (case["V"] + 2 * case["given"] + 1 + 2 * case["top"]), "flops": 0}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "place":
        new, lens = _placed(case)
        rot, page, near = case["rot"], case["page"], case["near"]
        freq = torch.tensor(s.freq or [], dtype=torch.float64, device="cuda")
        axis = torch.tensor(s.axis or [0] * (rot // 2), device="cuda")
        q_out, kp, vp = s.q_out.double(), s.k_pages.double(), s.v_pages.double()
        t0 = 0
        for b, (n, m) in enumerate(zip(new, lens)):
            at = torch.arange(m - n, m, device="cuda")
            own_pos = (at + s.first).view(n, 1) if s.pos is None else s.pos[t0:t0 + n]
            z = torch.polar(torch.ones(n, rot // 2, dtype=torch.float64, device="cuda"), own_pos[:, axis].double() * freq).unsqueeze(1) if rot else None

            def made(x, w):
                x = x[t0:t0 + n].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(dim=2, keepdim=True) + s.eps) * w.double()
                if rot:
                    head = x[..., :rot]
                    c = head.unflatten(2, (rot // 2, 2)) if near else head.unflatten(2, (2, rot // 2)).transpose(2, 3)
                    c = torch.view_as_real(torch.view_as_complex(c.contiguous()) * z)
                    x = torch.cat([(c if near else c.transpose(2, 3)).flatten(2), x[..., rot:]], dim=2)
                return x

            q_out[t0:t0 + n] = made(s.q, s.q_norm)
            pages = s.table[b].long()[at // page]
            kp[pages, at % page] = made(s.k, s.k_norm)
            vp[pages, at % page] = s.v[t0:t0 + n].double()
            t0 += n
        return q_out, kp, vp
    if case["op"] == "cross":
        new, mem = _memories(case)
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        G, t0, m0 = H // Hkv, 0, 0
        out = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
        for n, m in zip(new, mem):
            rows = torch.arange(m0, m0 + m, device="cuda")
            if s.keep is not None:
                rows = rows[s.keep[rows] != 0]
            if len(rows):
                for h in range(Hkv):
                    q = s.q[t0:t0 + n, h * G:(h + 1) * G].double()
                    p = torch.softmax(torch.einsum("ngd,kd->ngk", q, s.k[rows, h].double()) * D ** -0.5, dim=2)
                    out[t0:t0 + n, h * G:(h + 1) * G] = torch.einsum("ngk,kd->ngd", p, s.v[rows, h].double())
            t0, m0 = t0 + n, m0 + m
        return out
    rows, k = case["rows"], case["top"]
    lp = torch.zeros(rows, case["given"], dtype=torch.float64, device="cuda")
    H = torch.zeros(rows, dtype=torch.float64, device="cuda")
    top_lp = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    temps, given = s.temp.tolist(), s.given.tolist()
    for r in range(rows):
        l = s.logits[r].double()
        big = l.max()
        if big == -float("inf"):
            lw = l
        elif temps[r] > 0:
            lw = torch.log_softmax((l - big) / temps[r], dim=0)
        else:
            lw = torch.full_like(l, -float("inf"))
            lw[(l == big).nonzero()[0]] = 0
        some = lw > -float("inf")
        H[r] = -(lw[some].exp() * lw[some]).sum()
        if given[r]:
            tok = s.given[r].long()
            lp[r] = torch.where(tok >= 0, lw[tok.clamp(min=0)], torch.zeros_like(lp[r]))
        if k:
            top_lp[r] = lw.topk(k)[0]
    return lp, H, None, top_lp
