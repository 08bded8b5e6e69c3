"""Calls of one kernel: how their status word is cleared, and that they go on where the device holds no cluster of
their size (a partition with few SMs together).  The launchers' own text is compiled for the host against
a fake runtime whose largest cluster the test sets."""
import ctypes
import os
import subprocess

import pytest

from paper_2605_31105_gb300 import build as build_mod
from tests.host_block import _slice

HARNESS = r"""
#include <cuda_runtime_api.h>
#include <cstddef>
#include <cstdint>
#include <utility>
#define __host__
#define __device__
static int largest, launched, cluster_used, grid_used, memsets, clears, beside_used, solo_used, kernel_used;
static int attr_of(const cudaLaunchConfig_t* c, cudaLaunchAttributeID id) {
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == id)
      return id == cudaLaunchAttributeClusterDimension ? c->attrs[i].val.clusterDim.x : 1;
  return 0;
}
extern "C" cudaError_t cudaGetLastError() { return cudaSuccess; }
extern "C" cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { ++memsets; return cudaSuccess; }
template <class... P>
cudaError_t cudaOccupancyMaxActiveClusters(int* n, void (*)(P...), const cudaLaunchConfig_t* c) {
  *n = attr_of(c, cudaLaunchAttributeClusterDimension) <= largest ? 1 : 0;
  return cudaSuccess;
}
template <class... P, class... A>
cudaError_t cudaLaunchKernelEx(const cudaLaunchConfig_t* c, void (*k)(P...), A&&...);
namespace grkv {
static void count_launches(int) {}
%(launch)s
cudaError_t launch_clear_status(int*, cudaStream_t) { ++clears; return cudaSuccess; }
constexpr int kMaxSolo = 8;
%(call)s
constexpr int GRKV_F32 = 0, GRKV_BF16 = 1, kThreads = 256, kMmaThreads = 128, kMmaRows = 16;
struct AttendArgs { int U, g, t, cols; int* status; };
struct CacheShape { int U, g, t, cols, shift, dtype, simt; };
struct __nv_bfloat16 {};
template <class T, int R> void k_cross_few(const AttendArgs, int, bool) {}
template <int NT> void k_cross_mma(const AttendArgs, int, bool) {}
%(few)s
%(rule)s
void k_one(int, int*, int) {}
}
using namespace grkv;
static void note(int) {}
template <class T> static void note(const T&) {}
static int number(const AttendArgs& a) { return 0; }
template <class... P, class... A>
cudaError_t cudaLaunchKernelEx(const cudaLaunchConfig_t* c, void (*k)(P...), A&&... args) {
  const int cl = attr_of(c, cudaLaunchAttributeClusterDimension);
  cluster_used = cl ? cl : 1;
  if (cluster_used > largest || c->gridDim.x %% cluster_used) return cudaErrorInvalidClusterSize;
  ++launched;
  grid_used = c->gridDim.x;
  beside_used = attr_of(c, cudaLaunchAttributeProgrammaticStreamSerialization);
  const void* f = (const void*)k;
  kernel_used = f == (const void*)k_cross_mma<1> ? 101 : f == (const void*)k_cross_mma<2> ? 102 : 0;
  return cudaSuccess;
}
static void reset(int limit) { largest = limit; launched = memsets = clears = 0; }
extern "C" int call(long long blocks, long long bytes, int limit, int* out) {
  reset(limit);
  int word;
  const int rc = launch_call(k_one, blocks, 128, (size_t)bytes, &word, 0, 5);
  out[0] = cluster_used, out[1] = grid_used, out[2] = memsets, out[3] = clears, out[4] = beside_used, out[5] = launched;
  return rc;
}
extern "C" int cross(int U, int g, int t, int cols, int dtype, int limit, int simt, int* out) {
  reset(limit);
  const CacheShape s{U, g, t, cols, 4, dtype, simt};
  const AttendArgs a{U, g, t, cols, nullptr};
  out[6] = cross_is_few(s, 152);
  const int rc = out[6] ? launch_cross_few(s, a, 152, 0) : 0;
  out[0] = cluster_used, out[1] = grid_used, out[2] = memsets, out[3] = kernel_used, out[5] = launched;
  return rc;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    def text(name):
        with open(os.path.join(build_mod.CSRC, name)) as f:
            return f.read()

    common, rows, cross = (text(f) for f in ("grkv_internal.cuh", "cache_rows.cuh", "grkv_attend_cross.cu"))
    code = HARNESS % {
        "launch": _slice(common, "// chained: the work before this launch", "// Byte offsets of the workspace"),
        "call": _slice(rows, "constexpr size_t kLongCall", "inline Table table_of("),
        "few": _slice(cross, "cudaError_t launch_few(", "}  // namespace\n\n// CTAs of a unit"),
        "rule": _slice(cross, "static int few_ctas(", "}  // namespace grkv"),
    }
    tmp = str(tmp_path_factory.mktemp("calls"))
    src, so = os.path.join(tmp, "calls.cpp"), os.path.join(tmp, "calls.so")
    with open(src, "w") as f:
        f.write(code)
    cuda = os.path.dirname(os.path.dirname(build_mod.nvcc()))
    # (its own runtime calls, though another runtime may be loaded)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-w", "-I",
                    os.path.join(cuda, "include"), "-o",
                    so, src], check=True)
    return ctypes.CDLL(so)


def _call(lib, blocks, size, limit=8):
    out = (ctypes.c_int * 7)()
    assert lib.call(ctypes.c_longlong(blocks), ctypes.c_longlong(size), limit, out) == 0 and out[5] == 1
    return dict(zip(("cluster", "grid", "memsets", "clears", "beside"), out))


def test_status_of_a_call(lib):
    assert _call(lib, 1, 1 << 30) == dict(cluster=1, grid=1, memsets=0, clears=0, beside=0)
    for blocks in (2, 5, 8):
        assert _call(lib, blocks, 100) == dict(cluster=blocks, grid=blocks, memsets=0, clears=0, beside=0)
        assert _call(lib, blocks, 100, 1) == dict(cluster=1, grid=blocks, memsets=1, clears=0, beside=0)
        assert _call(lib, blocks, 1 << 30, 1) == dict(cluster=1, grid=blocks, memsets=0, clears=1, beside=1)
    assert _call(lib, 9, 100) == dict(cluster=1, grid=9, memsets=1, clears=0, beside=0)
    assert _call(lib, 9, 1 << 30) == dict(cluster=1, grid=9, memsets=0, clears=1, beside=1)


def _cross(lib, u, g, t, cols, dtype=1, limit=8, simt=0):
    out = (ctypes.c_int * 7)()
    assert lib.cross(u, g, t, cols, dtype, limit, simt, out) == 0
    if not out[6]:
        return None
    assert out[5] == 1
    return tuple(out)[:4]


def test_clusters_of_encoder_attention(lib):
    # cluster, grid (a cluster more where it scans the tables), memsets, kernel
    assert _cross(lib, 128, 1, 1, 95) == (2, 258, 0, 0)
    assert _cross(lib, 128, 1, 1, 95, limit=1) == (1, 128, 1, 0)      # 48 entries a thread: no scan
    assert _cross(lib, 1, 1, 1, 95) == (8, 8, 0, 0) and _cross(lib, 1, 1, 1, 95, limit=2) == (2, 2, 0, 0)
    assert _cross(lib, 32, 4, 1, 95) == (8, 264, 0, 101)
    assert _cross(lib, 32, 8, 2, 95) == (8, 264, 0, 102)
    assert _cross(lib, 32, 4, 1, 95, limit=4) == (4, 132, 0, 101)
    assert _cross(lib, 1, 1, 1, 1) == (1, 1, 0, 0) and _cross(lib, 3, 1, 1, 1) == (1, 4, 0, 0)
    assert _cross(lib, 64, 8, 1, 95, dtype=0) == (4, 260, 0, 0)


def test_calls_that_go_to_the_tiles(lib):
    for args in ((8, 17, 1, 10), (8, 1, 17, 10), (1, 1, 1, 2000), (128, 16, 1, 1000), (64, 64, 16, 1)):
        assert _cross(lib, *args) is None
    assert _cross(lib, 8, 9, 1, 10, dtype=0) is None and _cross(lib, 128, 8, 1, 95, dtype=0) is None
    assert _cross(lib, 1 << 28, 1, 1, 1) == (1, 1 << 28, 1, 0)        # the largest number of units
    assert _cross(lib, 1, 64, 1 << 22, 1) is None
    # the portable kernels' flag: CUDA cores only
    assert _cross(lib, 8, 3, 1, 10, simt=1) is None and _cross(lib, 8, 2, 1, 10, simt=1) == (2, 18, 0, 0)
