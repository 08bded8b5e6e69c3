// Where the new rows of every unit go: first rows, positions and slots of the pool, from the
// lengths and counts alone.
//
// A thread per row, blocks of whole units where a unit has up to 1024 rows.  Few bytes (12 a row) and
// little arithmetic: bound by the latency of a few dependent loads, count and length, then the table.
#include "cache_rows.cuh"

using namespace grkv;

namespace {

constexpr int kMapThreads = 1024;
constexpr int kMaxPackedUnits = 1 << 20;
constexpr int kOwnSums = 4096;   // units up to which each block adds up the counts of those before its own

struct MapArgs {
  RowMove m;
  const int32_t *table, *parent, *offset;
  int64_t* first_row;   // packed: first rows [U + 1], or null
  int32_t* pos;
  int64_t* slot;
  int per;              // rows of a block
  bool summed;          // first_row has been written
};

__device__ __forceinline__ int block_total(int x, int* sm) {
  x = __reduce_add_sync(0xffffffffu, x);
  __syncthreads();   // the last call's sums have been read
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = x;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, sm[threadIdx.x & 31]);
}

// Exclusive sum over the block's threads, and in *total the whole.
__device__ __forceinline__ int block_scan(int x, int* sm, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int scan = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += y;
  }
  __syncthreads();
  if (lane == 31) sm[warp] = scan;
  __syncthreads();
  const int sum = sm[lane];
  *total = __reduce_add_sync(0xffffffffu, sum);
  return __reduce_add_sync(0xffffffffu, lane < warp ? sum : 0) + scan - x;
}

// First rows of many units, by one block (counts are checked by k_cache_map).
__global__ void __launch_bounds__(kMapThreads) k_map_first(const int32_t* __restrict__ count, int U, int t,
                                                           int64_t* first_row) {
  __shared__ int sums[32];
  int before = 0;
  for (int u0 = 0; u0 < U; u0 += kMapThreads) {
    const int u = u0 + threadIdx.x;
    int all;
    const int at = block_scan(u >= U ? 0 : count ? min(max(count[u], 0), t) : t, sums, &all);
    if (u < U) first_row[u] = before + at;
    before += all;
  }
  if (threadIdx.x == 0) first_row[U] = before;
}

__global__ void __launch_bounds__(kMapThreads)
    k_cache_map(const __grid_constant__ MapArgs a, int* word, int solo) {
  __shared__ CallStatus::Smem shared;
  __shared__ int sums[32], firsts[kMapThreads + 1], up[2][kMapThreads], depth[2][kMapThreads];
  const CallStatus st(word, &shared, solo);
  RowMove m = a.m;
  m.status = st.at();
  const int tid = threadIdx.x, U = m.tb.U, t = m.t;
  const int rows = U * t, n0 = blockIdx.x * a.per, n = n0 + tid;
  const bool mine = tid < a.per && n < rows;
  const int u = mine ? n / t : 0, i = mine ? n - u * t : 0, u0 = n0 / t;
  const int cnt = mine ? rows_of(m, u) : 0;
  int first = u * t, total = rows;
  if (a.summed) {
    first = mine ? (int)a.first_row[u] : 0;
    total = (int)a.first_row[U];
  } else if (a.first_row) {
    // rows in front of the block's first unit, of all units, and in front of each of the block's
    int before = 0, all = 0;
    for (int x = tid; x < U; x += kMapThreads) {
      const int c = rows_of(m, x);
      all += c;
      if (x < u0) before += c;
    }
    before = block_total(before, sums);
    total = block_total(all, sums);
    const int mu = u0 + tid;   // a thread a unit: the block has up to 1024
    const int c = mu < U && mu * (int64_t)t < n0 + a.per ? rows_of(m, mu) : 0;
    int block;
    firsts[tid] = before + block_scan(c, sums, &block);
    __syncthreads();
    first = firsts[u - (mine ? u0 : 0)];
    if (mine && i == 0) a.first_row[u] = first;
    if (blockIdx.x == 0 && tid == 0) a.first_row[U] = total;
  }
  int ahead = i;   // of the unit's first new row, in positions
  if (a.parent) {
    // Depths by doubling: after round k a node knows its ancestor 2^k steps up and how many steps
    // there are to it.  (Whole units: t <= 256.)
    int y = -1;
    if (mine && i < cnt) {
      y = a.parent[n];
      if (y < -1 || y >= i) {
        set_status(m.status, GRKV_ERR_INVALID_ARG);
        y = -1;
      }
    }
    up[0][tid] = y < 0 ? -1 : tid - i + y;
    depth[0][tid] = y < 0 ? 0 : 1;
    int from = 0;
    for (int d = 1; d < t; d <<= 1, from ^= 1) {
      __syncthreads();
      const int x = up[from][tid];
      up[from ^ 1][tid] = x < 0 ? -1 : up[from][x];
      depth[from ^ 1][tid] = depth[from][tid] + (x < 0 ? 0 : depth[from][x]);
    }
    ahead = depth[from][tid];
  }
  if (mine) {
    const int64_t out = (int64_t)first + i;
    if (i < cnt) {
      const long long base = (long long)m.len[u] - cnt, s = base + i;
      const long long p = base + ahead + (a.offset ? a.offset[u] : 0);
      long long row = -1;
      if (s >= 0 && s < m.tb.cols << m.tb.shift) row = pool_row(m.tb, a.table, u, (int)s, m.status);
      else set_status(m.status, GRKV_ERR_INVALID_ARG);
      if (p < 0 || p > 0x7fffffff) set_status(m.status, GRKV_ERR_INVALID_ARG);
      a.pos[out] = p < 0 || p > 0x7fffffff ? -1 : (int)p;
      a.slot[out] = row;
    } else if (!a.first_row) {
      a.pos[out] = -1;
      a.slot[out] = -1;
    }
    if (a.first_row && n >= total) {
      a.pos[n] = -1;
      a.slot[n] = -1;
    }
  }
  st.end();
}

}  // namespace

extern "C" int grkv_cache_map(const grkv_cache_params* p, const int32_t* count, const int32_t* parent,
                              const int32_t* offset, const int32_t* table, const int32_t* len,
                              int64_t* first_row, int32_t* pos, int64_t* slot, void* ws,
                              size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (parent && s.t > kMaxTree) return GRKV_ERR_UNSUPPORTED;
  if (first_row && s.U > kMaxPackedUnits) return GRKV_ERR_UNSUPPORTED;
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({table, len, pos}, 4));
    GRKV_TRY(check_ptrs({slot}, 8));
  }
  GRKV_TRY(check_optional(count, 4));
  GRKV_TRY(check_optional(parent, 4));
  GRKV_TRY(check_optional(offset, 4));
  GRKV_TRY(check_optional(first_row, 8));
  cudaStream_t st = (cudaStream_t)stream;
  char* w = (char*)ws;
  if (s.U == 0) {
    GRKV_TRY(clear_status(w, L, st));
    return first_row ? cuda_rc(cudaMemsetAsync(first_row, 0, 8, st)) : GRKV_OK;
  }
  const int rows = s.U * s.t;
  const RowMove m{table_of(s), s.t, count, len, nullptr};
  const bool summed = first_row && s.U > kOwnSums;
  const MapArgs a{m, table, parent, offset, first_row, pos, slot,
                  s.t <= kMapThreads ? kMapThreads / s.t * s.t : kMapThreads, summed};
  if (summed) {
    count_launches(1);
    GRKV_TRY(cuda_rc(launch_kernel(false, 1, k_map_first, dim3(1), kMapThreads, 0, st, count, s.U, s.t, first_row)));
  }
  return cuda_rc(launch_call(k_cache_map, (rows + a.per - 1) / a.per, kMapThreads, (size_t)rows * 12, (int*)(w + L.status), st, a));
}
