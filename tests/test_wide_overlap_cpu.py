"""Outputs that overlap inputs: the host's test of tables against one byte by byte, and what the calls refuse (they look at addresses only)."""
import ctypes as C
import os
import random
import subprocess

import numpy as np
import pytest

EINVAL = -1
SOURCE = r"""
#include "tables.h"
extern "C" int overlap(uint64_t a, int64_t ra, int64_t la, int64_t na, uint64_t b, int64_t rb, int64_t lb, int64_t nb) {
    using namespace accerl;
    return share({(const void*)a, ra, la, na}, {(const void*)b, rb, lb, nb});
}
"""


def test_tables_against_their_bytes(tmp_path):
    from paper_2211_15023_amd import build
    (tmp_path / "t.cpp").write_text(SOURCE)
    subprocess.run([build.CXX, "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t.so")],
                   check=True)
    f = C.CDLL(str(tmp_path / "t.so")).overlap
    f.argtypes = [C.c_uint64] + [C.c_int64] * 3 + [C.c_uint64] + [C.c_int64] * 3
    rng = random.Random(7)
    seen = [0, 0]
    for i in range(20000):
        na, nb = rng.randint(1, 6), rng.randint(1, 6)
        la = na + rng.randint(0, 8)
        lb = max(nb, la) if rng.random() < 0.5 else nb + rng.randint(0, 8)
        a, ra, b, rb = rng.randint(100, 160), rng.randint(0, 6), rng.randint(100, 160), rng.randint(0, 6)
        both = {a + r * la + k for r in range(ra) for k in range(na)} & {b + r * lb + k for r in range(rb) for k in range(nb)}
        assert bool(f(a, ra, la, na, b, rb, lb, nb)) == bool(both), (a, ra, la, na, b, rb, lb, nb)
        seen[bool(both)] += 1
    assert min(seen) > 3000
    assert not f(1 << 20, 1 << 24, 1 << 62, 8, 16, 1 << 24, 1 << 62, 8)              # strides past 64 bits
    assert f(1 << 20, 1 << 24, 1 << 40, 8, (1 << 20) + (1 << 62), 4, 1 << 41, 8)


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def test_a_dense_layer_writes_over_none_of_its_inputs(A):
    lib = A.load_library()
    raw = np.zeros((1 << 17) + 256, np.uint8)
    p = (raw.ctypes.data + 255) // 256 * 256
    M, N, K = 3, 5, 100
    xq, sx, wq, sw, bias, out, work = (p + 8192 * i for i in range(7))
    n = A.accerl_dense_i8_workspace(M, K)
    last = out + (M - 1) * 64 * 2 + N * 2 - 2                                          # the last element of an output of rows 64 apart
    # xq sx wq sw bias M N K relu out dtype ld stream
    fixed = [xq, sx, wq, sw, bias, M, N, K, 0, out, 1, 64, None]
    for at, where in ((0, out), (0, last // 16 * 16), (1, out + 4), (1, last - 8), (2, out), (2, out - 2032), (3, out + 8), (3, last - 16), (4, out), (4, last - 12)):
        args = list(fixed)
        args[at] = where
        assert lib.accerl_dense_i8(*args) == EINVAL, (at, where - out)
        assert "overlap" in A.accerl_last_error()
    # x dtype ldx wq sw bias M N K relu out dtype ld ws bytes stream
    floating = [xq, 1, 128, wq, sw, bias, M, N, K, 0, out, 1, 64, work, n, None]
    for at, where in ((3, out), (4, out + 8), (5, last - 12), (13, out), (13, xq), (13, last // 16 * 16), (13, xq - n + 16)):
        args = list(floating)
        args[at] = where
        assert lib.accerl_dense_i8_dynamic(*args) == EINVAL, (at, where - out)
        assert "overlap" in A.accerl_last_error()
