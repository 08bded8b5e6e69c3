// Attention over encoder states for few rows (up to 16 a unit: single tokens) of caches that are small
// enough for a call to be a matter of latency.
//
// A cluster of CTAs takes a unit, its warps the unit's slots, 16 or 8 to a step, in turn: there is
// nothing to plan, no second kernel joins parts, and every warp keeps a whole step's K and V in flight,
// read straight to registers.  A lane holds 16 bytes of a row (8 dimensions of bf16: two slots side by side
// in a warp); the sums of a step's logits over the lanes are a transpose-reduction that leaves one logit
// to a lane.  References (running maximum, log2 units), sums and outputs of a CTA's warps are joined in
// its shared memory, those of the cluster's CTAs in the first one's, read from the others'.
#include <algorithm>

#include "attend_plan.cuh"

namespace grkv {
namespace {

using namespace sm100;

constexpr int kThreads = 256, kWarps = kThreads / 32;

template <typename T, int R>
struct Few {
  static constexpr int kDims = 16 / (int)sizeof(T);   // of a lane
  static constexpr int kLanes = kD / kDims;           // of a slot
  static constexpr int kSide = 32 / kLanes;           // slots side by side
  static constexpr int kLoad = R <= 4 ? 8 : 4;        // slots of a lane in a step; with R, up to kLanes logits
  static constexpr int kSlots = kSide * kLoad;        // of a step: 16 at most, in one page
  static constexpr int kStep = kLanes / (kLoad * R);  // lanes that end with the same logit
  static_assert(kStep >= 1, "a logit to a lane");
  struct Smem {
    int err;
    float ml[kWarps][R][2];
    float4 o[kWarps][R][kD / 4];
    float2 part_ml[R];          // of the CTA
    float4 part[R][kD / 4];
  };
};

// The 16 bytes of a lane as fp32.
__device__ __forceinline__ void widen(const uint4& x, float (&y)[4]) {
  y[0] = __uint_as_float(x.x);
  y[1] = __uint_as_float(x.y);
  y[2] = __uint_as_float(x.z);
  y[3] = __uint_as_float(x.w);
}
__device__ __forceinline__ void widen(const uint4& x, float (&y)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(w[i] << 16);
    y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Sums x[0..N) over groups of kLanes lanes; a lane ends with the sum of x[(lane % kLanes) N / kLanes].
template <int N, int kLanes>
__device__ __forceinline__ float sum_lanes(float (&x)[N], int lane) {
  int d = kLanes / 2;
#pragma unroll
  for (int n = N / 2; n >= 1; n /= 2, d /= 2) {
    const bool up = (lane & d) != 0;
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float send = up ? x[e] : x[e + n];
      x[e] = (up ? x[e + n] : x[e]) + __shfl_xor_sync(0xffffffffu, send, d);
    }
  }
#pragma unroll
  for (; d >= 1; d /= 2) x[0] += __shfl_xor_sync(0xffffffffu, x[0], d);
  return x[0];
}

__device__ __forceinline__ float4 ld_cluster(const float4* p, uint32_t rank) {
  float4 x;
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ float2 ld_cluster2(const float2* p, uint32_t rank) {
  float2 x;
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at) : "memory");
  return x;
}

__device__ __forceinline__ int ld_cluster1(const int* p, uint32_t rank) {
  int x;
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}

// The faults of a call's lengths, counts and pages, as the cluster in front of the units' looks for them, so
// that the status needs no clearing before the call (3 us of a call of 128 units).
__device__ __forceinline__ int scan_faults(const AttendArgs& a, int first, int step) {
  int err = 0;
  const int all = a.U * a.cols;
#pragma unroll 8
  for (int x = first; x < all; x += step) {
    const int u = x / a.cols, c = x - u * a.cols, L = unit_len(a, u), tokens = unit_tokens(a, u);
    if (c == 0 && (L != __ldg(a.len + u) || (a.qlen && tokens != __ldg(a.qlen + u)))) err = GRKV_ERR_INVALID_ARG;
    if (tokens > 0 && c << a.shift < L && (unsigned)__ldg(a.table + x) >= (unsigned)a.P) err = GRKV_ERR_INVALID_ARG;
  }
  return err;
}

// Before the first CTA reads the others' shared memory: what they wrote there is visible.
__device__ __forceinline__ void cluster_ready() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// After it, and before any of them may end.  x: a value made of everything that this thread read, so that the
// reads have returned (an arrival that is not a release, without it, let CTAs end under reads of them).
__device__ __forceinline__ void cluster_done(float x) {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::"f"(x) : "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The least of the CTAs' codes, in the first one (all threads).
__device__ __forceinline__ int cluster_min(int* err, int C, int rank) {
  if (C == 1) return *err;
  cluster_ready();
  const int x = rank == 0 && threadIdx.x < C ? ld_cluster1(err, threadIdx.x) : *err;
  __syncwarp();
  const int all = __reduce_min_sync(0xffffffffu, x);
  cluster_done(__int_as_float(all));
  return all;
}

// grid: U clusters of C, and, with `scan` (U > 1), in front of them one that writes the status
template <typename T, int R>
__global__ void __launch_bounds__(kThreads, R <= 4 ? 2 : 1)
    k_cross_few(const __grid_constant__ AttendArgs a, int C, bool scan) {
  using F = Few<T, R>;
  constexpr int kDims = F::kDims, kLanes = F::kLanes, kLoad = F::kLoad;
  __shared__ typename F::Smem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cluster = blockIdx.x / C, rank = blockIdx.x - cluster * C, u = cluster - scan, rows = a.g * a.t;
  const int side = lane / kLanes, off = lane % kLanes * kDims;
  const int mine = lane % kLanes / F::kStep, my_row = mine / kLoad, my_slot = mine % kLoad;
  if (tid == 0) sm.err = 0;
  __syncthreads();
  if (u < 0) {
    const int fault = scan_faults(a, rank * kThreads + tid, C * kThreads);
    if (fault) sm.err = fault;
    __syncthreads();
    const int all = cluster_min(&sm.err, C, rank);
    if (rank == 0 && tid == 0) *a.status = all;
    return;
  }
  const int L = unit_len(a, u), tokens = unit_tokens(a, u);
  int err = 0;
  if (L != __ldg(a.len + u) || (a.qlen && tokens != __ldg(a.qlen + u))) err = GRKV_ERR_INVALID_ARG;

  const int steps = tokens > 0 ? (L + F::kSlots - 1) / F::kSlots : 0;
  const int stride = C * kWarps;
  int k = rank * kWarps + warp;
  auto look_up = [&](int step) {
    return step < steps ? __ldg(a.table + (size_t)u * a.cols + (step * F::kSlots >> a.shift)) : 0;
  };
  // this lane's part of a step's slots (zeros behind the unit's last)
  auto load = [&](const void* pool, int step, int page, uint4 (&x)[kLoad]) {
    const int x0 = step * F::kSlots, left = L - x0 - side;
    const T* row = (const T*)pool + (((size_t)page << a.shift) + (x0 & ((1 << a.shift) - 1)) + side) * kD + off;
#pragma unroll
    for (int j = 0; j < kLoad; ++j)
      x[j] = F::kSide * j < left ? *(const uint4*)(row + (size_t)F::kSide * j * kD) : make_uint4(0, 0, 0, 0);
  };
  int entry = look_up(k);
  float q[R][kDims], o[R][kDims];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool has = r < rows;
    widen(has ? *(const uint4*)((const T*)a.q + ((size_t)u * rows + r) * kD + off) : make_uint4(0, 0, 0, 0), q[r]);
#pragma unroll
    for (int d = 0; d < kDims; ++d) o[r][d] = 0.f;
  }
  float m = -INFINITY, l = 0.f;   // of row my_row; l of this lane's slots alone
  for (; k < steps; k += stride) {
    int page = entry;
    if ((unsigned)page >= (unsigned)a.P) {
      err = GRKV_ERR_INVALID_ARG;
      page = 0;
    }
    entry = look_up(k + stride);
    // (the next step's K asked for here already: 12.2 us -> 13.1 for one row of 128 units, two sets of inputs in
    // turn, which L2 holds in part)
    uint4 kk[kLoad], vv[kLoad];
    load(a.k, k, page, kk);
    load(a.v, k, page, vv);
    float x[R * kLoad];
#pragma unroll
    for (int s = 0; s < kLoad; ++s) {
      float y[kDims];
      widen(kk[s], y);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float sum = q[r][0] * y[0];
#pragma unroll
        for (int d = 1; d < kDims; ++d) sum = fmaf(q[r][d], y[d], sum);
        x[r * kLoad + s] = sum;
      }
    }
    const float dot = sum_lanes<R * kLoad, kLanes>(x, lane);
    const bool see = F::kSide * my_slot < L - k * F::kSlots - side;
    const float logit = see ? logit_of(dot, a.sl2) : -INFINITY;
    float top = logit;
#pragma unroll
    for (int d = kLoad / 2; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d * F::kStep));
    if (F::kSide == 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, kLanes));
    const float M = fmaxf(m, top), ref = M == -INFINITY ? 0.f : M;
    const float keep = fast_exp2(m - ref), p = see ? prob_of(logit, ref) : 0.f;
    m = M;
    l = l * keep + p;
    const bool scale = __any_sync(0xffffffffu, keep != 1.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!scale) break;
      const float f = __shfl_sync(0xffffffffu, keep, r * kLoad * F::kStep);
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[r][d] *= f;
    }
#pragma unroll
    for (int s = 0; s < kLoad; ++s) {
      float y[kDims];
      widen(vv[s], y);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float w = __shfl_sync(0xffffffffu, p, side * kLanes + (r * kLoad + s) * F::kStep);
#pragma unroll
        for (int d = 0; d < kDims; ++d) o[r][d] = fmaf(w, y[d], o[r][d]);
      }
    }
  }
  if (err) sm.err = err;   // one code: whichever thread's

  // the warp's rows: their sums over the lanes and sides, outputs over the sides
#pragma unroll
  for (int d = kLoad / 2; d >= 1; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d * F::kStep);
  if (F::kSide == 2) {
    l += __shfl_xor_sync(0xffffffffu, l, kLanes);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[r][d] += __shfl_xor_sync(0xffffffffu, o[r][d], kLanes);
  }
  if (side == 0) {
    if (my_slot == 0 && lane % F::kStep == 0) {
      sm.ml[warp][my_row][0] = m;
      sm.ml[warp][my_row][1] = l;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int d = 0; d < kDims; d += 4)
        sm.o[warp][r][(off + d) / 4] = make_float4(o[r][d], o[r][d + 1], o[r][d + 2], o[r][d + 3]);
  }
  __syncthreads();
  // the CTA's, a thread four columns of a row (R 32 <= 256 threads)
  const int r = tid >> 5;
  float M = -INFINITY, sum = 0.f;
  err = sm.err;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float f, const float4& x) {
    y.x = fmaf(f, x.x, y.x);
    y.y = fmaf(f, x.y, y.y);
    y.z = fmaf(f, x.z, y.z);
    y.w = fmaf(f, x.w, y.w);
  };
  if (r < R) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.ml[w][r][0]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = weight_of(sm.ml[w][r][0], M);
      sum += f * sm.ml[w][r][1];
      add(f, sm.o[w][r][lane]);
    }
  }
  if (C > 1) {
    if (r < R) {
      sm.part[r][lane] = y;
      if (lane == 0) {
        sm.part_ml[r] = make_float2(M, sum);
      }
    }
    cluster_ready();
    if (rank == 0 && tid < C) err = ld_cluster1(&sm.err, tid);
    if (rank == 0 && r < R) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int c = 1; c < 8; ++c) {
        if (c >= C) break;
        ml[c] = ld_cluster2(&sm.part_ml[r], c);
        x[c] = ld_cluster(&sm.part[r][lane], c);
      }
      float top = M;
#pragma unroll
      for (int c = 1; c < 8; ++c)
        if (c < C) top = fmaxf(top, ml[c].x);
      const float f = weight_of(M, top);
      M = top;
      sum *= f;
      y = make_float4(y.x * f, y.y * f, y.z * f, y.w * f);
#pragma unroll
      for (int c = 1; c < 8; ++c) {
        if (c >= C) break;
        const float g = weight_of(ml[c].x, M);
        sum += g * ml[c].y;
        add(g, x[c]);
      }
    }
    __syncwarp();
    err = __reduce_min_sync(0xffffffffu, err);
    cluster_done(y.x + y.y + y.z + y.w + sum + M + __int_as_float(err));
  }
  if (rank == 0 && r < R && r < rows && r % a.t < tokens) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t dst = (size_t)u * rows + r;
    store_row4((T*)a.out + dst * kD + lane * 4, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
    if (a.lse && lane == 0) a.lse[dst] = row_lse(M, sum);
  }
  // one unit: its cluster writes the status whole; without a scan, faults go to the cleared word
  if (rank == 0 && tid < 32) {
    err = __reduce_min_sync(0xffffffffu, err);
    if (tid == 0) {
      if (a.U == 1) *a.status = err;
      else if (err && !scan) set_status(a.status, err);
    }
  }
}

// -------------------------------------------------- 3 to 16 rows of bf16: warp-level products
// More rows than a lane's FMAs keep up with go through m16n8k16 products of each warp's own 16 slots, whose
// operands are read from the cache straight into the fragments: a call waits for memory, and has nothing to
// fill the 128-row tiles and the pipeline of the tcgen05 kernel with.  The 16 side of a product are slots (S^T =
// K Q^T) and dimensions (O^T = V^T P^T), the 8 side rows, of which there are few: a product takes an SM's
// quarter some 44 cycles, and with the sides the other way round eight rows took twice as many.
// Fragments.  K: a lane's part of a slot are 16-byte chunks, so that the products' order of dimensions is not
// theirs, but the queries' is the same.  V: a lane reads the same chunk of its four slots and pairs them up by
// permutes; an output fragment's rows are a chunk's elements.  P goes from S^T's fragment to a right operand
// by a transposition of 8 x 8.  Up to eight rows P is multiplied in two parts, its bf16 and what that
// leaves, and all that is rounded is the output; with more, products bound the call, and P is rounded once.
constexpr int kMmaThreads = 128, kMmaWarps = kMmaThreads / 32, kMmaRows = 16;
template <int NT>   // row tiles of 8
struct MmaSmem {
  int err;
  float2 ml[kMmaWarps][8 * NT], part_ml[8 * NT];
  float4 o[kMmaWarps][8 * NT][kD / 4];   // the first warp's becomes the CTA's
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

// grid as k_cross_few's
template <int NT>
__global__ void __launch_bounds__(kMmaThreads, NT == 1 ? 4 : 3)
    k_cross_mma(const __grid_constant__ AttendArgs a, int C, bool scan) {
  __shared__ MmaSmem<NT> sm;
  typedef __nv_bfloat16 T;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cluster = blockIdx.x / C, rank = blockIdx.x - cluster * C, u = cluster - scan, rows = a.g * a.t;
  const int i = lane >> 2, c = lane & 3;   // a fragment's row (a right operand's column) and place in it
  if (tid == 0) sm.err = 0;
  __syncthreads();
  if (u < 0) {
    const int fault = scan_faults(a, rank * kMmaThreads + tid, C * kMmaThreads);
    if (fault) sm.err = fault;
    __syncthreads();
    const int all = cluster_min(&sm.err, C, rank);
    if (rank == 0 && tid == 0) *a.status = all;
    return;
  }
  const int L = unit_len(a, u), tokens = unit_tokens(a, u);
  int err = 0;
  if (L != __ldg(a.len + u) || (a.qlen && tokens != __ldg(a.qlen + u))) err = GRKV_ERR_INVALID_ARG;
  const int steps = tokens > 0 ? (L + 15) / 16 : 0, stride = C * kMmaWarps;
  int k = rank * kMmaWarps + warp;
  auto look_up = [&](int step) {
    return step < steps ? __ldg(a.table + (size_t)u * a.cols + (step * 16 >> a.shift)) : 0;
  };
  int entry = look_up(k);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 q[NT][4];   // row 8 x + i, chunks of 8 dimensions 4 j + c
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 8 * x + i;
      q[x][j] = r < rows ? *(const uint4*)((const T*)a.q + ((size_t)u * rows + r) * kD + (4 * j + c) * 8) : zero;
    }
  // of rows 8 x + 2 c + e: the output, dimension 64 (j / 4) + 8 i + 2 (j % 4) + h in o[x][j][2 h + e]; the
  // reference; the sum of this lane's slots
  float o[NT][8][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[x][j][e] = 0.f;
    m[x][0] = m[x][1] = -INFINITY;
    l[x][0] = l[x][1] = 0.f;
  }
  for (; k < steps; k += stride) {
    int page = entry;
    if ((unsigned)page >= (unsigned)a.P) {
      err = GRKV_ERR_INVALID_ARG;
      page = 0;
    }
    entry = look_up(k + stride);
    const int x0 = k * 16, n = L - x0;   // slots of the step that the unit has
    const size_t base = (((size_t)page << a.shift) + (x0 & ((1 << a.shift) - 1))) * kD;
    uint4 kk[2][4], vv[4][2];   // K of slots i, i + 8, chunks 4 j + c; V of slots 2 c + {0, 1, 8, 9}, chunks i, i + 8
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kk[t][j] = 8 * t + i < n ? *(const uint4*)((const T*)a.k + base + (8 * t + i) * kD + (4 * j + c) * 8) : zero;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int slot = 2 * c + (x & 1) + 8 * (x >> 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        vv[x][h] = slot < n ? *(const uint4*)((const T*)a.v + base + slot * kD + h * 64 + i * 8) : zero;
    }
    float s[NT][4];   // slots i (0, 1) and i + 8 (2, 3), rows 2 c + {0, 1}
#pragma unroll
    for (int x = 0; x < NT; ++x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[x][e] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < 4; w += 2)
          mma16816(s[x], word(kk[0][j], w), word(kk[1][j], w), word(kk[0][j], w + 1), word(kk[1][j], w + 1),
                   word(q[x][j], w), word(q[x][j], w + 1));
    }
    uint32_t hi[NT][2], lo[NT][2];   // P of slots 0-7 and 8-15: column i, slots 2 c + {0, 1}
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      float keep[2], p[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float x0 = i < n ? logit_of(s[x][e], a.sl2) : -INFINITY;
        const float x1 = i + 8 < n ? logit_of(s[x][2 + e], a.sl2) : -INFINITY;
        float top = fmaxf(x0, x1);
#pragma unroll
        for (int d = 4; d <= 16; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float M = fmaxf(m[x][e], top), ref = M == -INFINITY ? 0.f : M;
        keep[e] = fast_exp2(m[x][e] - ref);
        m[x][e] = M;
        p[e] = i < n ? prob_of(x0, ref) : 0.f;
        p[2 + e] = i + 8 < n ? prob_of(x1, ref) : 0.f;
        l[x][e] = l[x][e] * keep[e] + (p[e] + p[2 + e]);
      }
      if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x][j][e] *= keep[e & 1];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        hi[x][t] = pack_bf16(p[2 * t], p[2 * t + 1]);
        if (NT == 1)
          lo[x][t] = transposed8(pack_bf16(p[2 * t] - __uint_as_float(hi[x][t] << 16),
                                           p[2 * t + 1] - __uint_as_float(hi[x][t] & 0xffff0000u)));
        hi[x][t] = transposed8(hi[x][t]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int h = j >> 2, w = j & 3;   // elements 2 w, 2 w + 1 of chunks i + 8 h
      const uint32_t v[4] = {word(vv[0][h], w), word(vv[1][h], w), word(vv[2][h], w), word(vv[3][h], w)};
      const uint32_t a0 = __byte_perm(v[0], v[1], 0x5410), a1 = __byte_perm(v[0], v[1], 0x7632);
      const uint32_t a2 = __byte_perm(v[2], v[3], 0x5410), a3 = __byte_perm(v[2], v[3], 0x7632);
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        mma16816(o[x][j], a0, a1, a2, a3, hi[x][0], hi[x][1]);
        if (NT == 1) mma16816(o[x][j], a0, a1, a2, a3, lo[x][0], lo[x][1]);
      }
    }
  }
  if (err) sm.err = err;

  // the warp's rows
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d <= 16; d *= 2) l[x][e] += __shfl_xor_sync(0xffffffffu, l[x][e], d);
      const int r = 8 * x + 2 * c + e;
      if (r >= rows) continue;
      if (i == 0) sm.ml[warp][r] = make_float2(m[x][e], l[x][e]);
#pragma unroll
      for (int j = 0; j < 8; j += 2)
        sm.o[warp][r][16 * (j >> 2) + 2 * i + (j >> 1 & 1)] =
            make_float4(o[x][j][e], o[x][j][2 + e], o[x][j + 1][e], o[x][j + 1][2 + e]);
    }
  __syncthreads();
  err = sm.err;
  auto add = [](float4* y, float f, const float4& x) {
    y->x = fmaf(f, x.x, y->x);
    y->y = fmaf(f, x.y, y->y);
    y->z = fmaf(f, x.z, y->z);
    y->w = fmaf(f, x.w, y->w);
  };
  auto store = [&](int r, const float4& y, float M, float sum) {
    if (r % a.t >= tokens) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t dst = (size_t)u * rows + r;
    store_row4((T*)a.out + dst * kD + lane * 4, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
    if (a.lse && lane == 0) a.lse[dst] = row_lse(M, sum);
  };
  // the CTA's, a warp a row
  for (int r = warp; r < rows; r += kMmaWarps) {
    float M = -INFINITY, sum = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kMmaWarps; ++w) M = fmaxf(M, sm.ml[w][r].x);
#pragma unroll
    for (int w = 0; w < kMmaWarps; ++w) {
      const float f = weight_of(sm.ml[w][r].x, M);
      sum += f * sm.ml[w][r].y;
      add(&y, f, sm.o[w][r][lane]);
    }
    if (C == 1) {
      store(r, y, M, sum);
      continue;
    }
    sm.o[0][r][lane] = y;
    if (lane == 0) sm.part_ml[r] = make_float2(M, sum);
  }
  if (C > 1) {
    cluster_ready();
    float used = 0.f;
    if (rank == 0 && tid < C) err = ld_cluster1(&sm.err, tid);
    for (int r = warp; rank == 0 && r < rows; r += kMmaWarps) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        if (z >= C) break;
        ml[z] = ld_cluster2(&sm.part_ml[r], z);
        x[z] = ld_cluster(&sm.o[0][r][lane], z);
      }
      float M = -INFINITY, sum = 0.f;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int z = 0; z < 8; ++z)
        if (z < C) M = fmaxf(M, ml[z].x);
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        if (z >= C) break;
        const float f = weight_of(ml[z].x, M);
        sum += f * ml[z].y;
        add(&y, f, x[z]);
      }
      store(r, y, M, sum);
      used += y.x + y.y + y.z + y.w + sum;
    }
    __syncwarp();
    err = __reduce_min_sync(0xffffffffu, err);
    cluster_done(used + __int_as_float(err));
  }
  if (rank == 0 && tid == 0) {
    if (a.U == 1) *a.status = err;
    else if (err && !scan) set_status(a.status, err);
  }
}

cudaError_t launch_few(const AttendArgs& a, bool f32, int C, cudaStream_t st) {
  const int rows = a.g * a.t;
  auto go = [&](auto kern, int threads) {
    while (C > 1 && !cluster_fits(C, kern, threads, 0)) C /= 2;
    // the scan of a call's tables takes less than the call: up to 32 entries a thread
    const bool scan = a.U > 1 && (int64_t)a.U * a.cols <= (int64_t)32 * C * threads;
    if (a.U > 1 && !scan) {
      const cudaError_t e = cudaMemsetAsync(a.status, 0, 4, st);
      if (e != cudaSuccess) return e;
    }
    count_launches(1);
    return launch_kernel(false, C, kern, dim3((unsigned)(a.U + scan) * (unsigned)C), threads, 0, st, a, C, scan);
  };
  if (f32)
    return rows == 1   ? go(k_cross_few<float, 1>, kThreads)
           : rows == 2 ? go(k_cross_few<float, 2>, kThreads)
           : rows <= 4 ? go(k_cross_few<float, 4>, kThreads)
                       : go(k_cross_few<float, 8>, kThreads);
  if (rows <= 2)
    return rows == 1 ? go(k_cross_few<__nv_bfloat16, 1>, kThreads) : go(k_cross_few<__nv_bfloat16, 2>, kThreads);
  return rows <= 8 ? go(k_cross_mma<1>, kMmaThreads) : go(k_cross_mma<2>, kMmaThreads);
}

}  // namespace

// CTAs of a unit, 128 slots each at least: up to three times the SMs in all, four times those of four warps.  An SM
// holds two of k_cross_few's at once (one of fp32 with 5 to 8 rows), four of k_cross_mma's (three with 9 rows and more),
// so a call of the most CTAs takes more than a wave; the rule below was measured with it.
static int few_ctas(const CacheShape& s, int sms) {
  const int most = (s.dtype == GRKV_BF16 && s.g * s.t > 2 ? 4 : 3) * sms;
  int C = 1;
  while (C < 8 && (int64_t)s.U * C * 2 <= most && (int64_t)s.cols << s.shift > 128 * C) C *= 2;
  return C;
}

// Whether a cluster a unit is faster than runs that are even over the SMs, by the slots that units can have (the
// host does not know their lengths): a CTA's run of them may be longer than an SM's even share by what planning
// and joining take, 10 us, less where rows make a slot dearer; many rows are bound by the products.  us in a
// graph, three sets of inputs in turn, the other kernels' behind the slash (`n`: units of n / 16 to n slots, `n-`: all
// of n):
//   bf16, 1 row    128 x 1500 14.5/24.5, 1 x 8000 9.5/12.0, 1 x 20000 18.5/13.3, 128 x 16000 108/107, 128 x 30000- 281/329
//         2 rows   128 x 1500 16.0/25.3, 64 x 6000 24.8/33.5, 128 x 16000 121/107
//         4        128 x 1500 16.3/24.9, 8 x 8000 14.6/20.5, 1 x 8000 14.5/13.3, 128 x 16000- 163/183, 512 x 8000 240/202
//         16       64 x 1500 20.3/21.7, 128 x 1500 26.4/26.3, 64 x 6000 39.7/34.5
//   fp32, 1        128 x 1500 22.6/28.5, 1 x 8000 12.3/11.1, 64 x 6000 39.1/45.1
//         4        64 x 1500 15.8/21.7, 128 x 1500 27.8/28.9, 1 x 8000 19.3/12.1
//         8        64 x 1500 28.9/31.5, 128 x 1500 47.9/42.2
bool cross_is_few(const CacheShape& s, int sms) {
  const int rows = s.t <= 16 ? s.g * s.t : 17, C = few_ctas(s, sms);
  const int64_t cap = (int64_t)s.cols << s.shift, run = cap / C, share = s.U * cap / sms;
  if (s.dtype == GRKV_F32)
    return rows <= 2 ? run <= 800 + share / 2 : rows <= 4 ? run <= 800 : rows <= 8 && run <= 400;
  if (s.simt && rows > 2) return false;   // CUDA cores, and P in fp32
  return rows == 1   ? run <= 1700 + share
         : rows == 2 ? run <= 1000 + share / 2
         : rows <= 8 ? run <= 900 + share / 4
                     : rows <= kMmaRows && run <= 1000 && share <= 1500;
}

cudaError_t launch_cross_few(const CacheShape& s, const AttendArgs& a, int sms, cudaStream_t st) {
  return launch_few(a, s.dtype == GRKV_F32, few_ctas(s, sms), st);
}

}  // namespace grkv
