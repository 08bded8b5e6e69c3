// Attention over encoder states for few rows (up to 8 a unit: single tokens) of caches that are small
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
  static constexpr int kLoad = R <= 4 ? 8 : 4;        // slots of a lane in a step
  static constexpr int kSlots = kSide * kLoad;        // of a step: 16 at most, in one page
  static constexpr int kSum = kLoad * R <= kLanes ? kLoad : kLanes / R;   // whose logits are summed at once
  static constexpr int kStep = kLanes / (kSum * R);   // lanes that end with the same logit
  struct Smem {
    int err;
    float ml[kWarps][R][2];
    float4 o[kWarps][R][kD / 4];
    float part_ml[R][2];        // of the CTA
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

__device__ __forceinline__ float4 ld_cluster(const void* p, uint32_t rank) {
  float4 x;
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ float2 ld_cluster2(const void* p, uint32_t rank) {
  float2 x;
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at) : "memory");
  return x;
}

__device__ __forceinline__ int ld_cluster1(const void* p, uint32_t rank) {
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
  constexpr int kDims = F::kDims, kLanes = F::kLanes, kSum = F::kSum;
  __shared__ typename F::Smem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cluster = blockIdx.x / C, rank = blockIdx.x - cluster * C, u = cluster - scan, rows = a.g * a.t;
  const int side = lane / kLanes, off = lane % kLanes * kDims;
  const int mine = lane % kLanes / F::kStep, my_row = mine / kSum, my_slot = mine % kSum;
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
    const int x0 = k * F::kSlots;
    const size_t row = (((size_t)page << a.shift) + (x0 & ((1 << a.shift) - 1)) + side) * kD + off;
    uint4 kk[F::kLoad], vv[F::kLoad];
    const int n = L - x0 - side;   // slots of the lane's side that the unit has: those F::kSide j < n
#pragma unroll
    for (int j = 0; j < F::kLoad; ++j)
      kk[j] = F::kSide * j < n ? *(const uint4*)((const T*)a.k + row + (size_t)F::kSide * j * kD) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < F::kLoad; ++j)
      vv[j] = F::kSide * j < n ? *(const uint4*)((const T*)a.v + row + (size_t)F::kSide * j * kD) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j0 = 0; j0 < F::kLoad; j0 += kSum) {
      float x[R * kSum];
#pragma unroll
      for (int s = 0; s < kSum; ++s) {
        float y[kDims];
        widen(kk[j0 + s], y);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float sum = q[r][0] * y[0];
#pragma unroll
          for (int d = 1; d < kDims; ++d) sum = fmaf(q[r][d], y[d], sum);
          x[r * kSum + s] = sum;
        }
      }
      const float dot = sum_lanes<R * kSum, kLanes>(x, lane);
      const bool see = F::kSide * (j0 + my_slot) < n;
      const float logit = see ? dot * a.sl2 : -INFINITY;
      float top = logit;
#pragma unroll
      for (int d = kSum / 2; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d * F::kStep));
      if (F::kSide == 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, kLanes));
      const float M = fmaxf(m, top), ref = M == -INFINITY ? 0.f : M;
      const float keep = fast_exp2(m - ref), p = see ? fast_exp2(logit - ref) : 0.f;
      m = M;
      l = l * keep + p;
      const bool scale = __any_sync(0xffffffffu, keep != 1.f);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (!scale) break;
        const float f = __shfl_sync(0xffffffffu, keep, r * kSum * F::kStep);
#pragma unroll
        for (int d = 0; d < kDims; ++d) o[r][d] *= f;
      }
#pragma unroll
      for (int s = 0; s < kSum; ++s) {
        float y[kDims];
        widen(vv[j0 + s], y);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float w = __shfl_sync(0xffffffffu, p, side * kLanes + (r * kSum + s) * F::kStep);
#pragma unroll
          for (int d = 0; d < kDims; ++d) o[r][d] = fmaf(w, y[d], o[r][d]);
        }
      }
    }
  }
  if (err) sm.err = err;   // one code: whichever thread's

  // the warp's rows: their sums over the lanes and sides, outputs over the sides
#pragma unroll
  for (int d = kSum / 2; d >= 1; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d * F::kStep);
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
        sm.part_ml[r][0] = M;
        sm.part_ml[r][1] = sum;
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
        ml[c] = ld_cluster2(sm.part_ml[r], c);
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

template <typename T>
cudaError_t launch_few(const AttendArgs& a, int C, bool scan, cudaStream_t st) {
  const int rows = a.g * a.t;
  auto go = [&](auto kern) {
    count_launches(1);
    return launch_kernel(false, C, kern, dim3((unsigned)(a.U + scan) * (unsigned)C), kThreads, 0, st, a, C, scan);
  };
  return rows == 1 ? go(k_cross_few<T, 1>) : rows == 2 ? go(k_cross_few<T, 2>)
         : rows <= 4 ? go(k_cross_few<T, 4>) : go(k_cross_few<T, 8>);
}

}  // namespace

// CTAs of a unit: three to an SM in all, 128 slots each at least.
static int few_ctas(const CacheShape& s, int sms) {
  int C = 1;
  while (C < 8 && (int64_t)s.U * C * 2 <= 3 * sms && (int64_t)s.cols << s.shift > 128 * C) C *= 2;
  return C;
}

// Whether a cluster a unit is faster than runs that are even over the SMs, by the slots that the units
// can have (the host does not know their lengths).  One or two rows: a CTA's run may be longer than an SM's even
// share by what planning and joining take.  bf16, 128 units of up to 1500 slots 12.0 us for 24.0, of 30000
// 281 for 329 (194 for 186 where their lengths lie between 1900 and 30000), one of 8000 9.5 for 11.9, of 20000 18.5 for
// 13.3; fp32 22.6 for 28.5, one of 8000 12.3 for 11.1.  More rows are bound by issue: four of bf16 over 64
// units of 1500 14.8 for 17.4, over 128 27.1 for 25.0; eight over 32 units of 400 7.2 for 12.7, of 1500 19.9 for 16.7;
// fp32 four over 128 units of 1500 27.8 for 28.9, eight over 64 28.9 for 31.5, over 128 47.9 for 42.2.
bool cross_is_few(const CacheShape& s, int sms) {
  const int rows = s.t <= 8 ? s.g * s.t : 9, C = few_ctas(s, sms);
  const int64_t cap = (int64_t)s.cols << s.shift, run = cap / C, share = s.U * cap / sms;
  const bool f32 = s.dtype == GRKV_F32;
  if (rows <= 2) return f32 ? run <= 800 + share / 2 : run <= 1700 + share;
  if (rows <= 4) return run <= (f32 ? 800 : 400);
  return rows <= 8 && (f32 ? run <= 400 : run <= 200 && s.U * C <= sms);
}

cudaError_t launch_cross_few(const CacheShape& s, const AttendArgs& a, int sms, cudaStream_t st) {
  const int C = few_ctas(s, sms);
  // the scan of a call's tables takes less than the call: up to 32 entries a thread
  const bool scan = s.U > 1 && (int64_t)s.U * s.cols <= (int64_t)32 * C * kThreads;
  if (s.U > 1 && !scan) {
    const cudaError_t e = cudaMemsetAsync(a.status, 0, 4, st);
    if (e != cudaSuccess) return e;
  }
  return s.dtype == GRKV_F32 ? launch_few<float>(a, C, scan, st) : launch_few<__nv_bfloat16>(a, C, scan, st);
}

}  // namespace grkv
