"""What the serving calls' host code hands to the kernels, without a GPU (wt_serve.cpp over recording stand-ins)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2608_12114_gb300 import build, wt

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("serve") / "host.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", cuda, os.path.join(HERE, "_serve_host.cpp"),
                    os.path.join(build.CSRC, "wt_serve.cpp"), "-o", so], check=True)
    L = C.CDLL(so)
    L.host_error.restype = C.c_char_p
    L.host_place.restype = C.POINTER(wt.PlaceDesc)
    L.host_reset()
    return L


AT = 1 << 40  # buffers nobody reads, 2^36 bytes apart


def buffers(n):
    return [AT + (i << 36) for i in range(n)]


def place(parts, **kw):
    q, k, v, q_out, k_pages, v_pages, begin, table, lens, turns = buffers(10)
    d = wt.PlaceDesc(begin=begin, table=table, len=lens, turns=turns, q_stride=256, k_stride=128, v_stride=128, out_stride=256, table_stride=4,
                     in_dtype=wt.WT_F32, dtype=wt.WT_BF16, n_req=1, n_tokens=3, heads=4, kv_heads=2, head_dim=64, rot_dim=64, page=16,
                     n_pages=8, max_len=60)
    if "q" in parts:
        d.q, d.q_out = q, q_out
    if "k" in parts:
        d.k, d.k_pages = k, k_pages
    if "v" in parts:
        d.v, d.v_pages = v, v_pages
    for name, x in kw.items():
        setattr(d, name, x)
    return d


def test_values_alone_are_not_turned(L):
    """Without q and k nothing is turned: whatever stands in turns, pos, their pitch and axes does not reach the kernel."""
    for kw in (dict(turns=None), dict(turns=AT + 4), dict(turns=None, pos=AT + 2, pos_stride=-7, axes=200), dict(first_pos=-3)):
        d = place("v", **kw)
        d.axis[5] = 250
        L.host_reset()
        assert L.wt_place(None, C.byref(d), None) == wt.WT_OK, L.host_error()
        got = L.host_place().contents
        assert L.host_launches() == 1 and got.v == d.v
        assert got.rot_dim == 0 and not got.turns and not got.pos
    for parts in ("q", "k", "qk", "kv", "qkv"):  # which the others look at
        assert L.wt_place(None, C.byref(place(parts, turns=None)), None) == wt.WT_EINVAL and b"turns" in L.host_error()
        d = place(parts)
        L.host_reset()
        assert L.wt_place(None, C.byref(d), None) == wt.WT_OK and L.host_place().contents.rot_dim == 64
        assert L.host_place().contents.turns == d.turns


def test_row_tiles_up_to_2_31_rows(L):
    """wt_cross takes n_tokens * heads up to 2^31 - 1; a tile of 8, 16, 32 or up to 256 rows may end past that."""
    for G in (1, 2, 3, 7, 65, 127, 128):
        for rows in (8, 16, 32, 2 * (128 // G * G)):
            most = (2 ** 31 - 1) // G
            for n in (0, 1, rows // G, rows // G + 1, most - 1, most):
                if n <= 2 ** 30:
                    assert L.host_row_tiles(n, G, rows) == -(-n * G // rows), (n, G, rows)
