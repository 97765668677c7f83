"""What the serving calls' host code hands to the kernels, without a GPU (wt_serve.cpp over recording stand-ins)."""
import ctypes as C
import os
import random
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


def test_a_merge_has_parts_of_two_ctas(L):
    """wt_cross launches its merge where a memory may have more than one cell; its grid is a CTA less than the parts' own."""
    r = random.Random(1)
    merged = 0
    for _ in range(2000):
        kv, G, D = r.choice((1, 2, 3, 4, 8)), r.choice((1, 2, 7, 128)), r.choice((8, 64, 72, 128))
        q, k, v, begin, mem_begin, mem_len = buffers(6)
        tokens, states = r.choice((1, 2, 9, 33, 700)), r.choice((1, 15, 16, 17, 32, 64, 65, 128, 129, 70000))
        d = wt.CrossDesc(q=q, out=q, begin=begin, k=k, v=v, mem_begin=mem_begin, mem_len=mem_len, q_stride=kv * G * D, out_stride=kv * G * D,
                         mem_stride=kv * D, mem_head=D, n_mem=states, dtype=r.choice((wt.WT_BF16, wt.WT_F16)), n_req=r.choice((1, 2, 50)),
                         n_tokens=tokens, max_new=r.choice((1, tokens)), max_mem=r.choice((0, 1, states, 2 * states)), heads=kv * G,
                         kv_heads=kv, head_dim=D, scale=r.choice((0.1, 0.0, -1.0)))
        L.host_reset()
        assert L.wt_cross(None, C.byref(d), None) == wt.WT_OK, L.host_error()
        assert L.host_launches() == L.host_counted() in (1, 2)
        if L.host_launches() == 2:
            merged += 1
            assert L.host_cross_ctas() >= 2
    assert merged > 50  # one in ten memories is long, and half of the calls bound theirs by it
