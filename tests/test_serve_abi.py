"""The serving calls without a GPU: structures, constants, and what is refused before any CUDA call."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2608_12114_gb300 import build, wt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wt_serve.h")
STRUCTS = {"wt_adapt_desc": wt.AdaptDesc, "wt_attend_desc": wt.AttendDesc, "wt_probs_desc": wt.ProbsDesc,
           "wt_verify_desc": wt.VerifyDesc}


@pytest.fixture(scope="module")
def L():
    build.build()
    return wt.lib()


def test_structures_match_the_header(tmp_path):
    """Every field's offset and every structure's size, as a C compiler sees them."""
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
    for name in ("WT_ADAPT_MAX_RANK", "WT_ADAPT_MAX_SLOTS", "WT_VERIFY_MAX_VOCAB"):
        v = re.search(r"#define %s \(?([0-9]+)(?: << ([0-9]+))?\)?" % name, src)
        assert int(v.group(1)) << int(v.group(2) or 0) == getattr(wt, name)


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "%s"\nint main(void) { return 0; }\n' % HEADER)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-fsyntax-only", str(src)], check=True)


def test_null_and_host_only_handles_are_refused(L):
    with wt.Handle([], wt.WT_OPEN_HOST_ONLY) as h:
        for call, args in (("wt_adapt", (wt.AdaptDesc(), 1)), ("wt_attend", (wt.AttendDesc(),)), ("wt_probs", (wt.ProbsDesc(),)),
                           ("wt_verify", (wt.VerifyDesc(),))):
            a = [C.byref(args[0])] + list(args[1:])
            assert getattr(L, call)(None, *a, None) == wt.WT_EINVAL and call in L.wt_last_error().decode()
            assert getattr(L, call)(h.ptr, *a, None) == wt.WT_ENOTSUP and call in L.wt_last_error().decode()
