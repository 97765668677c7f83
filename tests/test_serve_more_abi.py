"""Placing, attention to memories and log probabilities without a GPU: structures, constants, turns, and what is refused before any CUDA call."""
import ctypes as C
import math
import os
import re
import subprocess
from fractions import Fraction

import pytest

from paper_2608_12114_gb300 import build, wt
from tests import _serve_more

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wt_serve.h")
STRUCTS = {"wt_place_desc": wt.PlaceDesc, "wt_cross_desc": wt.CrossDesc, "wt_logprobs_desc": wt.LogprobsDesc}


@pytest.fixture(scope="module")
def L():
    build.build()
    return wt.lib()


def test_structures_match_the_header(tmp_path):
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "%s"' % HEADER, "int main(void) {"]
    for name, s in STRUCTS.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f[0], name, f[0]) for f in s._fields_]
    src = tmp_path / "s.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "s")], check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True).stdout.splitlines())
    for name, s in STRUCTS.items():
        assert int(got[name]) == C.sizeof(s)
        for f in s._fields_:
            assert int(got["%s.%s" % (name, f[0])]) == getattr(s, f[0]).offset, (name, f[0])


def test_constants_match_the_header():
    src = open(HEADER).read()
    for name in ("WT_PLACE_MAX_DIM", "WT_PLACE_MAX_AXES", "WT_PLACE_NEIGHBOURS", "WT_LOGPROBS_MAX_TOP"):
        assert int(re.search(r"#define %s (\d+)" % name, src).group(1)) == getattr(wt, name)


def test_null_and_host_only_handles_are_refused(L):
    with wt.Handle([], wt.WT_OPEN_HOST_ONLY) as h:
        for call, d in (("wt_place", wt.PlaceDesc()), ("wt_cross", wt.CrossDesc()), ("wt_logprobs", wt.LogprobsDesc())):
            assert getattr(L, call)(None, C.byref(d), None) == wt.WT_EINVAL and call in L.wt_last_error().decode()
            assert getattr(L, call)(h.ptr, C.byref(d), None) == wt.WT_ENOTSUP and call in L.wt_last_error().decode()


def test_turns_are_fractions_of_a_turn():
    """In the kernel's integers: the angle of any position is its true one modulo a turn, up to half a unit of
    turns for each position and the 32 bits that are kept."""
    from paper_2608_12114_gb300 import serving
    freq = [1.0, 0.5, 10000.0 ** -0.3, 2 * math.pi, 7.0, -0.25, 1e-9, 0.0]
    turns = serving.turns(freq, device="cpu").tolist()
    for f, t in zip(freq, turns):
        for pos in (0, 1, 1000, 2 ** 20 + 7, 2 ** 30, -(2 ** 31), 2 ** 31 - 1):
            top = ((pos * t) % 2 ** 64) >> 32
            got = (top - 2 ** 32 if top >= 2 ** 31 else top) / 2 ** 32 * 2 * math.pi
            off = (got - _serve_more.angle(pos, f)) / (2 * math.pi)
            off -= round(off)
            assert -2.0 ** -32 - 2.0 ** -33 - 1e-15 <= off <= 2.0 ** -33 + 1e-15, (f, pos, off)
    assert turns[-1] == 0 and turns[5] < 0
    assert Fraction(turns[0]) == round(Fraction(2 ** 64) / (2 * Fraction(31415926535897932384626433832795028841971, 10 ** 40)))
    for bad in (float("nan"), float("inf")):
        with pytest.raises(ValueError):
            serving.turns([bad], device="cpu")
