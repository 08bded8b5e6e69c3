"""Cosine and sine of fractions of a turn (fp32 rows): the kernels' own text, compiled for the host, against 64 bits."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2605_31105_gb300 import build as build_mod
from tests.host_block import _slice

HARNESS = r"""
#include <cmath>
#include <cstdint>
#include <cstring>
#define __device__
#define __forceinline__ inline
static float __uint_as_float(uint32_t x) { float y; memcpy(&y, &x, 4); return y; }
static uint32_t __float_as_uint(float x) { uint32_t y; memcpy(&y, &x, 4); return y; }
%s
extern "C" void run(int n, const uint32_t* f, float* c, float* s) {
  for (int i = 0; i < n; ++i) cos_sin(f[i], c + i, s + i);
}
"""


@pytest.fixture(scope="module")
def cos_sin(tmp_path_factory):
    with open(os.path.join(build_mod.CSRC, "rope.cuh")) as f:
        text = _slice(f.read(), "__device__ __forceinline__ void cos_sin(", "// bf16: the special function unit")
    tmp = str(tmp_path_factory.mktemp("angles"))
    src, so = os.path.join(tmp, "a.cpp"), os.path.join(tmp, "a.so")
    with open(src, "w") as f:
        f.write(HARNESS % text)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-fPIC", "-shared", "-o", so, src], check=True)
    lib = ctypes.CDLL(so)

    def run(f):
        f = np.ascontiguousarray(f, np.uint32)
        c, s = np.empty(f.shape, np.float32), np.empty(f.shape, np.float32)
        ptr = lambda x: x.ctypes.data_as(ctypes.c_void_p)
        lib.run(f.size, ptr(f), ptr(c), ptr(s))
        return c.astype(np.float64), s.astype(np.float64)
    return run


# The header's bound for fp32 rows, 2^-23: of the angle 7.5e-8 radians at most (conversion 2^-28 turns, the constant
# 2^-25 of pi / 4, the product 2^-25), of the polynomials' steps some 2^-25 each, the last at half a step of 1.
def test_cosines_and_sines(cos_sin):
    eighths = (np.arange(8, dtype=np.uint64)[:, None] << 29) + np.arange(-2000, 2001)[None].astype(np.uint64)
    f = np.concatenate([(eighths & 0xffffffff).ravel(),
                        np.random.default_rng(0).integers(0, 1 << 32, 1 << 21, dtype=np.uint64)])
    c, s = cos_sin(f)
    # angles to 2^-50 of an eighth: the whole eighths are taken out first
    k = (f + (1 << 28)) >> np.uint64(29)
    rest = (f.astype(np.int64) - (k.astype(np.int64) << 29)) * (2 * np.pi / 2.0 ** 32)
    h = np.sqrt(0.5)
    ck, sk = np.array([1, h, 0, -h, -1, -h, 0, h, 1])[k], np.array([0, h, 1, h, 0, -h, -1, -h, 0])[k]
    assert np.abs(c - (ck * np.cos(rest) - sk * np.sin(rest))).max() <= 2.0 ** -23
    assert np.abs(s - (sk * np.cos(rest) + ck * np.sin(rest))).max() <= 2.0 ** -23


def test_quarters_are_exact(cos_sin):
    c, s = cos_sin([0, 1 << 30, 1 << 31, 3 << 30])
    assert c.tolist() == [1, 0, -1, 0] and s.tolist() == [0, 1, 0, -1]
