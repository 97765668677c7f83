"""One step of several requests over one checkpoint, as a serving program makes it.

A one-layer decoder is written, opened and ingested.  Its requests share a prompt whose keys and
values are in hand, have a paged cache of their own, an adapter each (or none), and a few drafted
tokens.  The step then

  projects     every token with wt_pass (up to 16 activation columns), wt_adapt beside it;
  places       the queries, and the new keys and values in their requests' pages (wt_place);
  attends      to the shared prompt and each request's own keys (wt_attend);
  answers      with the head's logits, their probabilities at each request's temperature (wt_probs),
               the tokens that stay (wt_verify), and the log probability of every token that was given
               or drafted, with the likeliest others (wt_logprobs).

    python examples/serving_step.py
"""
import os
import sys
import tempfile

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2608_12114_gb300 import pipeline, serving, synth, wt  # noqa: E402

HEADS, DIM, PAGE = 20, 128, 16


class Decoder:
    """A decoder layer and head in device memory, with the calls of one step."""

    def __init__(self, h: wt.Handle):
        self.h = h
        mats = pipeline.matrices(h)
        self.dev = pipeline.DeviceCheckpoint.allocate(h, mats)
        self.dev.adopt(h, stream=self.stream)
        self.k = {mats.name(k): k for k in range(len(mats))}

    @property
    def stream(self) -> int:
        return torch.cuda.current_stream().cuda_stream

    def weight(self, name: str) -> torch.Tensor:
        m = self.dev.mats[self.k[name]]
        return self.dev.bufs[self.k[name]].view(torch.bfloat16).view(m.shape)

    def project(self, names, x: torch.Tensor):
        """[x W^T for each matrix], fp32: one wt_pass, every weight read once for all tokens."""
        T, K = x.shape
        ws = [self.weight(n) for n in names]
        ys = [torch.empty(T, w.shape[0], device="cuda") for w in ws]
        self.h.pass_([wt.gemv_desc(w.data_ptr(), wt.WT_BF16, w.shape[0], K, x.data_ptr(), y.data_ptr(), cols=T)
                      for w, y in zip(ws, ys)], self.stream)
        return ys


def norm(x: torch.Tensor) -> torch.Tensor:
    return (x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6)).to(torch.bfloat16).contiguous()


def step(m: Decoder, tokens, begin, slot, adapters, prefix, cache, table, lens, temperature, q, u, u_draw):
    """One step: `tokens` holds each request's last token and its drafts, begin where each request's
    tokens start, lens its own keys including theirs.  Returns every tensor that the step makes."""
    T, B = len(tokens), len(lens)
    counts = begin.diff().tolist()
    d = HEADS * DIM
    x = m.weight("embed")[tokens.long()].float()
    xn = norm(x)
    yq, yk, yv = m.project(["layers.0.q", "layers.0.k", "layers.0.v"], xn)
    m.h.adapt([serving.adapters(xn, y, slot, *adapters[n]) for n, y in (("q", yq), ("v", yv))], m.stream)
    # the new tokens' keys and values go to their pages
    of = torch.repeat_interleave(torch.arange(B), torch.tensor(counts)).cuda()
    qs = torch.empty(T, HEADS, DIM, dtype=torch.bfloat16, device="cuda")
    heads = [y.view(T, HEADS, DIM) for y in (yq, yk, yv)]
    m.h.place(serving.placement(begin, cache[0], cache[1], table, lens, q=heads[0], q_out=qs, k=heads[1], v=heads[2],
                                max_len=int(lens.max())), m.stream)
    att = torch.empty_like(qs)
    m.h.attend(serving.attention(qs, att, begin, cache[0], cache[1], table, lens, max_new=max(counts),
                                 max_len=int(lens.max()), prefix_k=prefix[0], prefix_v=prefix[1]), m.stream)
    (yo,) = m.project(["layers.0.o"], att.view(T, d))
    x = x + yo
    xn2 = norm(x)
    gate, up = m.project(["layers.0.gate", "layers.0.up"], xn2)
    (down,) = m.project(["layers.0.down"], (torch.nn.functional.silu(gate) * up).to(torch.bfloat16))
    xf = norm(x + down)
    (logits,) = m.project(["lm_head"], xf)
    p = torch.empty_like(logits)
    m.h.probs(serving.probabilities(logits, p, temperature=temperature[of]), m.stream)
    # the drafts are all but each request's first token
    drafted = torch.cat([tokens[int(b) + 1:int(b) + c] for b, c in zip(begin[:-1], counts)])
    dbegin = begin - torch.arange(B + 1, dtype=torch.int32, device="cuda")
    accepted = torch.empty(B, dtype=torch.int32, device="cuda")
    out = torch.empty(B, max(counts), dtype=torch.int32, device="cuda")
    m.h.verify(serving.verification(p, drafted, dbegin, u, u_draw, accepted, out, q=q), m.stream)
    # what the target gives each token's successor: a draft's, or none
    given = torch.cat([torch.cat([tokens[int(b) + 1:int(b) + c], tokens.new_full((1,), -1)]) for b, c in zip(begin[:-1], counts)])
    lp, top, top_lp = torch.empty(T, 1, device="cuda"), torch.empty(T, 5, dtype=torch.int32, device="cuda"), torch.empty(T, 5, device="cuda")
    m.h.logprobs(serving.log_probabilities(logits, given=given.view(T, 1), given_lp=lp, top=top, top_lp=top_lp,
                                           temperature=temperature[of]), m.stream)
    return dict(xn=xn, yq=yq, yv=yv, q=qs, att=att, yo=yo, logits=logits, p=p, drafted=drafted, dbegin=dbegin,
                accepted=accepted, tokens=out, given=given, lp=lp, top=top, top_lp=top_lp)


def inputs(vocab: int, d: int, seed: int = 0, counts=(4, 1, 6), prompt: int = 700, own=(20, 55, 9), slots: int = 3, rank: int = 16):
    """A batch of requests: sizes as a small server has them, values from the seed."""
    g = torch.Generator("cuda").manual_seed(seed)
    B, T = len(counts), sum(counts)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, device="cuda", generator=g) * std).to(dtype)

    lens = torch.tensor([n + c for n, c in zip(own, counts)], dtype=torch.int32, device="cuda")
    most = -(-int(lens.max()) // PAGE)
    table = torch.randperm(B * most, device="cuda", generator=g).view(B, most).int()
    return dict(
        tokens=torch.randint(0, vocab, (T,), dtype=torch.int32, device="cuda", generator=g),
        begin=torch.tensor([sum(counts[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda"),
        # the first request has no adapter
        slot=torch.repeat_interleave(torch.arange(B, dtype=torch.int32) % slots - 1, torch.tensor(counts)).int().cuda(),
        adapters={n: (normal(slots, rank, d, std=d ** -0.5), normal(slots, d, rank, std=0.05),
                      torch.full((slots,), 2.0, device="cuda")) for n in "qv"},
        prefix=(normal(prompt, HEADS, DIM), normal(prompt, HEADS, DIM)),
        cache=(normal(B * most, PAGE, HEADS, DIM), normal(B * most, PAGE, HEADS, DIM)),
        table=table, lens=lens, temperature=torch.tensor([0.7, 0.0, 1.0], device="cuda")[:B],
        q=torch.softmax(normal(T - B, vocab, dtype=torch.float32), dim=1),
        u=torch.rand(T - B, device="cuda", generator=g), u_draw=torch.rand(B, device="cuda", generator=g))


def main():
    with tempfile.TemporaryDirectory() as tmp:
        ck = synth.build("mid", tmp, layers=1, vocab=4096)
        with wt.Handle(ck.paths) as h:
            m = Decoder(h)
            r = step(m, **inputs(4096, HEADS * DIM))
            torch.cuda.synchronize()
            for b, (n, t) in enumerate(zip(r["accepted"].tolist(), r["tokens"].tolist())):
                print("request %d: %d drafted tokens stay; tokens %s" % (b, n, t[:n + 1]))
            print("status %d, %d kernels" % (h.device_status(), h.kernel_launches()))


if __name__ == "__main__":
    main()
