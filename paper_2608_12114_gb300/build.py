"""Builds libwt.so in-tree for sm_103a (nvcc for the kernels, the host compiler for the C ABI)."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libwt.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
SOURCES = ["wt_kernels.cu", "wt_fnv.cu", "wt_cols.cu", "wt_umma.cu", "wt_q8rows.cu", "wt_colshort.cu", "wt_host.cpp", "wt_dlpack.cpp",
           "wt_noalloc.cu", "wt_serve.cpp", "wt_adapt.cu", "wt_attend.cu", "wt_prefix.cu", "wt_draw.cu", "wt_place.cu", "wt_cross.cu", "wt_crosswide.cu", "wt_logprobs.cu"]
HEADERS = ["wt_cross.cuh", "wt_tmem.cuh", "wt_kernels.h", "wt_fnv.h", "wt_q8rows.h", "wt_device.cuh", "wt_serve.h", "wt_serve.cuh", os.path.join("..", "..", "include", "wt.h"),
           os.path.join("..", "..", "include", "wt_dlpack.h"), os.path.join("..", "..", "include", "wt_serve.h")]


def _nvcc():
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    raise RuntimeError("nvcc not found")


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    nvcc = _nvcc()
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O2,-Wall,-fvisibility=hidden"]

    def compile_one(src):
        obj = os.path.join(bdir, src + ".o")
        cmd = [nvcc] + ARCH + common + ["-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cu"):
            cmd += ["-Xptxas", "-v"] if verbose else []
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("compile failed: %s\n%s%s" % (" ".join(cmd), r.stdout, r.stderr))
        if verbose:
            sys.stderr.write(r.stdout + r.stderr)
        return obj

    with ThreadPoolExecutor(len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc] + ARCH + ["-shared", "-o", tmp] + objs + ["-lpthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed: %s\n%s%s" % (" ".join(cmd), r.stdout, r.stderr))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
