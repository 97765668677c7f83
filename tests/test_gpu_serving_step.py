"""examples/serving_step.py: the whole step against the same step in 64 bits, and in a graph."""
import os
import sys

import pytest

from paper_2608_12114_gb300 import build, synth, wt
from tests import _serve

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    build.build()
    wt.lib()
    return torch


def test_the_step_matches_64_bits(torch, tmp_path):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
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
        # each product against 64-bit sums of the same operands: 2e-3 of sum |W x|, as for the passes
        for n, y, x in (("q", r["yq"], r["xn"]), ("v", r["yv"], r["xn"]), ("o", r["yo"], r["att"].view(len(a["tokens"]), -1))):
            W, X = m.weight("layers.0." + n).double(), x.double()
            want = X @ W.t()
            if n in "qv":
                A, B, c = a["adapters"][n]
                want, s1, s2 = _serve.adapt(x, a["slot"], A, B, c, None, want)
                want, size = want.cuda(), (X.abs() @ W.t().abs()) + s2.cuda()
            else:
                size = X.abs() @ W.t().abs()
            assert ((y.double() - want).abs() <= 2e-3 * size).all(), n
        out, mag, qk = _serve.attend(r["q"], a["begin"], *a["prefix"], *a["cache"], a["table"], a["lens"], ex.DIM ** -0.5)
        tol = (2.0 ** -8 + 2.0 ** -18 * qk + 2.0 ** -15) * mag + 2.0 ** -8 * out.abs()
        assert ((r["att"].double().cpu() - out).abs() <= tol).all()
        of = torch.repeat_interleave(torch.arange(3), a["begin"].diff().cpu().long()).cuda()
        t = a["temperature"][of].double().view(-1, 1)
        l = r["logits"].double()
        p = torch.where(t > 0, torch.softmax(l / t.clamp(min=1e-9), dim=1), (l == l.amax(dim=1, keepdim=True)).double())
        assert ((r["p"].double() - p).abs() <= 1e-5 * p + 1e-9).all()
        want = _serve.verify(r["p"], a["q"], r["drafted"], r["dbegin"], a["u"], a["u_draw"], r["tokens"].shape[1] - 1)
        assert (r["accepted"].tolist(), r["tokens"].tolist()) == want


def test_the_example_runs(torch, capsys):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import serving_step as ex
    finally:
        sys.path.pop(0)
    ex.main()
    out = capsys.readouterr().out
    assert "request 2" in out and "status 0" in out
