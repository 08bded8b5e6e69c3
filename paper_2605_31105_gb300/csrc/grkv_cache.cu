// The paged cache: entry points of the page operators and of the attention that reads
// the pages, and the page operators' kernels.
//
// All of them move whole rows (256 bytes of bf16, 512 of fp32) or small integers: they
// are bound by memory or, for the tables, by latency.  The bookkeeping is deterministic:
// free pages are handed out from the lowest, units and columns ascending.
#include <algorithm>
#include <cmath>

#include "cache_rows.cuh"

using namespace grkv;

namespace {

int make_cache_shape(const grkv_cache_params* p, CacheShape* s) {
  if (!p) return GRKV_ERR_INVALID_ARG;
  if (p->units < 0 || p->group < 1 || p->d < 1 || p->pages < 1 || p->page < 1 ||
      p->max_pages < 1 || p->tokens < 1 || p->window < 0 || p->n_sink < 0)
    return GRKV_ERR_INVALID_ARG;
  if (!(p->scale >= 0.f) || std::isinf(p->scale)) return GRKV_ERR_INVALID_ARG;
  if (p->dtype != GRKV_F32 && p->dtype != GRKV_BF16) return GRKV_ERR_INVALID_ARG;
  if (p->flags & ~(GRKV_FORCE_SIMT | GRKV_TEST_TIMEOUT)) return GRKV_ERR_INVALID_ARG;
  if (p->d != kD || p->group > kMaxCacheGroup) return GRKV_ERR_UNSUPPORTED;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128)
    return GRKV_ERR_UNSUPPORTED;
  // pages, slots of a unit, entries of a table and rows of a call stay within 32-bit integers
  // (rows in two steps: U g t itself may pass 64 bits)
  if (p->pages > 1 << 30) return GRKV_ERR_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page > (int64_t)1 << 28) return GRKV_ERR_UNSUPPORTED;
  if (p->tokens > 1 << 28 || (int64_t)p->units * p->max_pages > (int64_t)1 << 30 ||
      (int64_t)p->units * p->group > (int64_t)1 << 28 ||
      (int64_t)p->units * p->group * p->tokens > (int64_t)1 << 28)
    return GRKV_ERR_UNSUPPORTED;
  s->U = p->units;
  s->g = p->group;
  s->t = p->tokens;
  s->P = p->pages;
  s->page = p->page;
  s->shift = p->page == 16 ? 4 : p->page == 32 ? 5 : p->page == 64 ? 6 : 7;
  s->cols = p->max_pages;
  s->W = std::min(p->window, 1 << 29);
  s->s = std::min(p->n_sink, 1 << 29);
  s->dtype = p->dtype;
  s->simt = (p->flags & GRKV_FORCE_SIMT) ? 1 : 0;
  s->test_timeout = (p->flags & GRKV_TEST_TIMEOUT) ? 1 : 0;
  s->scale = p->scale != 0.f ? p->scale : (float)(1.0 / std::sqrt((double)p->d));
  return GRKV_OK;
}

CacheWs plan_cache_ws(const CacheShape& s) {
  CacheWs L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align256(off + bytes);
    return at;
  };
  const size_t rows = attend_part_rows(s);   // of the parts of all CTAs
  L.status = take(256);
  L.rec = take((size_t)2 * kMaxAttendSms * 16);
  L.pml = take(rows * sizeof(float2));
  L.po = take(rows * kD * sizeof(float));
  // a reserve and an attention call do not need their parts at the same time
  const size_t attend = off;
  off = L.rec;
  L.list = take((size_t)s.P * 4);
  L.jobs = take((size_t)s.U * 16);
  L.total = std::max(attend, off);
  return L;
}

}  // namespace

namespace grkv {

int cache_begin(const grkv_cache_params* p, const void* ws, size_t ws_bytes, CacheShape* s, CacheWs* L) {
  GRKV_TRY(make_cache_shape(p, s));
  *L = plan_cache_ws(*s);
  GRKV_TRY(check_ptrs({ws}, 16));
  return ws_bytes < L->total ? GRKV_ERR_WORKSPACE_TOO_SMALL : GRKV_OK;
}

}  // namespace grkv

namespace {

__global__ void k_clear_status(int* word) {
  asm volatile("griddepcontrol.launch_dependents;");
  *word = 0;
}

// ------------------------------------------------------------------- fork, trim
// A thread per table entry.
__global__ void __launch_bounds__(1024)
    k_cache_fork(Table tb, int units_in, const int32_t* __restrict__ src,
                 const int32_t* __restrict__ table_in, const int32_t* __restrict__ len_in,
                 int32_t* table_out, int32_t* len_out, int32_t* refs, int* word, bool solo) {
  __shared__ int shared;
  const Status st(word, &shared, solo);
  const int all = tb.U * tb.cols;
  for (int x = blockIdx.x * blockDim.x + threadIdx.x; x < all; x += gridDim.x * blockDim.x) {
    const int u = x / tb.cols, c = x - u * tb.cols;
    int s = src[u];
    if (s < -1 || s >= units_in) {
      set_status(st.at, GRKV_ERR_INVALID_ARG);
      s = -1;
    }
    const int len = s >= 0 ? tb.clamped(len_in[s], st.at) : 0;
    int e = -1;
    if (c << tb.shift < len) {
      e = max(table_in[(size_t)s * tb.cols + c], -1);   // a column may be without a page
      if (e >= tb.P) {
        set_status(st.at, GRKV_ERR_INVALID_ARG);
        e = -1;
      }
      if (e >= 0) atomicAdd(refs + e, 1);
    }
    table_out[x] = e;
    if (c == 0) len_out[u] = len;
  }
  st.end();
}

__global__ void __launch_bounds__(1024)
    k_cache_trim(Table tb, int32_t* table, const int32_t* __restrict__ len, int32_t* refs, int* word,
                 bool solo) {
  __shared__ int shared;
  const Status st(word, &shared, solo);
  const int all = tb.U * tb.cols;
  for (int x = blockIdx.x * blockDim.x + threadIdx.x; x < all; x += gridDim.x * blockDim.x) {
    const int u = x / tb.cols, c = x - u * tb.cols, n = tb.clamped(len[u], st.at);
    if (c << tb.shift < n) continue;
    const int e = table[x];
    if (e < 0) continue;
    if (e >= tb.P) {
      set_status(st.at, GRKV_ERR_INVALID_ARG);
    } else if (atomicSub(refs + e, 1) <= 0) {   // nobody held it: the count stays
      atomicAdd(refs + e, 1);
      set_status(st.at, GRKV_ERR_INVALID_ARG);
    }
    table[x] = -1;
  }
  st.end();
}

// ---------------------------------------------------------------------- reserve
constexpr int kReserveThreads = 1024;

// Sum over the block before this thread, and in *total the whole.
__device__ __forceinline__ int block_scan(int x, int* total, int* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int scan = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += y;
  }
  __syncthreads();   // the last call's sums have been read
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) {
    const int y = warp_sum[w];
    if (w < warp) before += y;
    all += y;
  }
  *total = all;
  return before + scan - x;
}

// One block.  The columns that unit u is to write are [len / page, ceil(want / page)); one
// needs a new page if it has none or one that others hold too.  The decisions are all made
// on the counts as the call found them, before any of them changes: where every unit has a
// thread of its own and at most 32 such columns (a few tokens of every unit of a batch) they
// stay in that thread's registers, else they are marked in the table, -2 - page.  One column of 256
// units takes 9 us.  A unit's columns are one thread's work, three dependent loads each: the first
// reserve of 256 units of 2048 slots in pages of 16 takes 182 us, of 32768 slots 2.5 ms.
constexpr int kListShared = 4096;   // free pages that fit the block's own list
__global__ void __launch_bounds__(kReserveThreads)
    k_cache_reserve(Table tb, int32_t* table, const int32_t* __restrict__ len,
                    const int32_t* __restrict__ want, int32_t* refs, int32_t* list_ws, int4* jobs,
                    int* word) {
  __shared__ int warp_sum[32], shared, list_sm[kListShared];
  __shared__ uint32_t free_words[kReserveThreads / 2];   // a bit a page, 16 a thread
  const int tid = threadIdx.x, n = blockDim.x;
  // Marks which of the 16 K pages from p0 on nobody holds (read after a barrier).
  auto look = [&](int p0) {
    const int lane = tid & 31, a = p0 + (tid >> 5) * 512 + lane;
    int held[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) held[k] = a + k * 32 < tb.P ? refs[a + k * 32] : 1;
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const uint32_t w = __ballot_sync(0xffffffffu, held[k] <= 0);
      if (lane == k) mine = w;
    }
    if (lane < 16) free_words[(tid >> 5) * 16 + lane] = mine;
  };
  look(0);
  const Status st(word, &shared, true);
  const int per = (tb.U + n - 1) / n, u0 = min(tb.U, tid * per), u1 = min(tb.U, u0 + per);
  auto columns = [&](int u, int* c0, int* c1) {
    const int a = tb.clamped(len[u], st.at), b = tb.clamped(want[u], st.at);
    *c0 = a >> tb.shift;
    *c1 = b > a ? (b + tb.page() - 1) >> tb.shift : *c0;
    return a;
  };
  int mine = 0;
  uint32_t bits = 0;   // of the thread's only unit: columns from c0 on that need a page
  bool wide = per > 1;
  for (int u = u0; u < u1; ++u) {
    int c0, c1;
    columns(u, &c0, &c1);
    wide |= c1 - c0 > 32;
    for (int c = c0; c < c1; ++c) {
      const int e = table[(size_t)u * tb.cols + c];
      if (e >= tb.P) set_status(st.at, GRKV_ERR_INVALID_ARG);
      if (e < 0 || e >= tb.P || refs[e] > 1) {
        ++mine;
        bits |= 1u << ((c - c0) & 31);
      }
    }
  }
  const bool marks = __syncthreads_or(wide);
  int need;
  int at = block_scan(mine, &need, warp_sum);
  int32_t* list = need <= kListShared ? list_sm : list_ws;
  // the lowest free pages
  int found = 0;
  for (int p0 = 0; p0 < tb.P && found < need; p0 += n * 16) {
    const int a = p0 + tid * 16;
    if (p0 > 0) {
      __syncthreads();
      look(p0);
      __syncthreads();
    }
    uint32_t free_bits = (free_words[tid >> 1] >> (16 * (tid & 1))) & 0xffffu;
    int all, r = found + block_scan(__popc(free_bits), &all, warp_sum);
    for (; free_bits && r < need; free_bits &= free_bits - 1) list[r++] = a + __ffs(free_bits) - 1;
    found += all;
  }
  const bool enough = found >= need;
  if (!enough && tid == 0) set_status(st.at, GRKV_ERR_NO_PAGES);
  __syncthreads();
  if (enough && marks) {
    for (int u = u0; u < u1; ++u) {
      int c0, c1;
      columns(u, &c0, &c1);
      for (int c = c0; c < c1; ++c) {
        int32_t* e = table + (size_t)u * tb.cols + c;
        if (*e < 0 || *e >= tb.P)
          *e = -1;
        else if (refs[*e] > 1)
          *e = -2 - *e;
      }
    }
  }
  if (marks) __syncthreads();
  for (int u = u0; u < u1; ++u) {
    int4 job = make_int4(-1, -1, 0, 0);
    int c0, c1;
    const int a = columns(u, &c0, &c1);
    for (int c = c0; enough && c < c1; ++c) {
      int32_t* e = table + (size_t)u * tb.cols + c;
      int old = *e;   // the page to replace, or negative
      if (marks) {
        if (old >= 0) continue;
        old = old <= -2 ? -2 - old : -1;
      } else {
        if (!((bits >> (c - c0)) & 1)) continue;
        if (old >= tb.P) old = -1;
      }
      const int page = list[at++];
      refs[page] = 1;
      if (old >= 0) {
        const int part = a - (c << tb.shift);
        atomicSub(refs + old, 1);
        if (part > 0) job = make_int4(old, page, part, 0);
      }
      *e = page;
    }
    jobs[u] = job;
  }
  st.end();
}

// Copies the filled slots of the shared pages that a reserve replaced.
__global__ void k_cache_copy(int U, int row16, int page, const int4* __restrict__ jobs, uint4* k,
                             uint4* v) {
  chain_wait();
  for (int u = blockIdx.x; u < U; u += gridDim.x) {
    const int4 job = jobs[u];
    if (job.x < 0) continue;
    const size_t from = (size_t)job.x * page * row16, to = (size_t)job.y * page * row16;
    for (int i = threadIdx.x; i < job.z * row16; i += blockDim.x) {
      k[to + i] = k[from + i];
      v[to + i] = v[from + i];
    }
  }
}

// --------------------------------------------------------------- append, compact
// Copies of rows: a block takes 2 x 128 / kRow16 rows of one unit (grid (blocks of rows, units)),
// kRow16 lanes a row of kRow16 16-byte chunks, two rows of K and V in flight to a thread.  Bound
// by memory: 524288 kept rows of K and V (537 MB read and written, rows of 256 bytes from
// anywhere) in 90 us, 6.0 TB/s.  Those are read once and written for later (kOnce), which loads
// and stores say (95 us without; only one of the two 107 to 117).  256 threads 98 us, with
// four or eight rows each 101 and 131.
constexpr int kMoveThreads = 128, kMoveUnroll = 2;
constexpr int move_rows(int row16) { return kMoveUnroll * kMoveThreads / row16; }

// where(u, i, n, len, &from, &to): source and destination row of row i of unit u's n; false: none
template <int kRow16, bool kOnce, typename Where>
__device__ __forceinline__ void move_block(const RowMove& m, const uint4* k_in, const uint4* v_in,
                                           uint4* k, uint4* v, Where where) {
  const int ch = threadIdx.x % kRow16, r = threadIdx.x / kRow16;
  for (int u = blockIdx.y; u < m.tb.U; u += gridDim.y) {
    const int len = m.tb.clamped(m.len[u], m.status);
    const int n = rows_of(m, u), i0 = blockIdx.x * move_rows(kRow16) + r;
    long long to[kMoveUnroll];
    uint4 x[kMoveUnroll], y[kMoveUnroll];
#pragma unroll
    for (int j = 0; j < kMoveUnroll; ++j) {
      const int i = i0 + j * (kMoveThreads / kRow16);
      long long from = 0;
      to[j] = -1;
      if (i >= n || !where(u, i, n, len, &from, &to[j])) {
        to[j] = -1;
        continue;
      }
      const uint4 *pk = k_in + from * kRow16 + ch, *pv = v_in + from * kRow16 + ch;
      x[j] = kOnce ? __ldcs(pk) : *pk;
      y[j] = kOnce ? __ldcs(pv) : *pv;
    }
#pragma unroll
    for (int j = 0; j < kMoveUnroll; ++j) {
      if (to[j] < 0) continue;
      uint4 *pk = k + to[j] * kRow16 + ch, *pv = v + to[j] * kRow16 + ch;
      if (kOnce) {
        __stcs(pk, x[j]);
        __stcs(pv, y[j]);
      } else {
        *pk = x[j];
        *pv = y[j];
      }
    }
  }
}

template <int kRow16>
__global__ void __launch_bounds__(kMoveThreads)
    k_cache_append(RowMove m, const uint4* __restrict__ k_new, const uint4* __restrict__ v_new,
                   const int64_t* __restrict__ first, long long new_rows,
                   const int32_t* __restrict__ table, uint4* k, uint4* v) {
  move_block<kRow16, false>(m, k_new, v_new, k, v, [&](int u, int i, int n, int, long long* from,
                                                long long* to) {
    // the length as it is: clamped to the table, rows behind it would go over those before
    const long long slot = (long long)m.len[u] - n + i;
    const long long f = first ? first[u] : (long long)u * m.t;
    if (slot < 0 || slot >= m.tb.cols << m.tb.shift || f < 0 || f > new_rows - 1 - i) {
      set_status(m.status, GRKV_ERR_INVALID_ARG);
      return false;
    }
    *from = f + i;
    *to = pool_row(m.tb, table, u, (int)slot, m.status);
    return *to >= 0;
  });
}

// To other pages: every row by itself.
template <int kRow16>
__global__ void __launch_bounds__(kMoveThreads)
    k_cache_gather(RowMove m, const int32_t* __restrict__ idx, const int32_t* __restrict__ table_in,
                   const int32_t* __restrict__ table_out, const int32_t* __restrict__ first, uint4* k,
                   uint4* v) {
  move_block<kRow16, true>(m, k, v, k, v, [&](int u, int i, int, int len, long long* from, long long* to) {
    return kept_row(m, idx, table_in, len, table_out, first, false, u, i, from, to);
  });
}

// In place: a row only moves down, so chunks of rows in ascending order, each read as a whole
// before it is written, never overwrite a row that is still to be read.  A block owns 64
// bytes of every row of one unit's keys or values (grid (U, 2, row bytes / 64)).  Bound by the
// latency of a chunk's loads: 16384 of 32768 slots of 8 units 220 us (64 blocks), 4096 of
// 8192 of 64 units 88 us, 2048 of 32768 of 256 units 167 us (to other pages 90).
constexpr int kShiftThreads = 256, kShiftUnroll = 4;
template <int kRow16>
__global__ void __launch_bounds__(kShiftThreads)
    k_cache_shift(RowMove m, const int32_t* __restrict__ idx, const int32_t* __restrict__ table,
                  const int32_t* __restrict__ first, uint4* k, uint4* v) {
  const int u = blockIdx.x, ch = blockIdx.z * 4 + (threadIdx.x & 3), r0 = threadIdx.x >> 2;
  uint4* pool = blockIdx.y ? v : k;
  const int n = rows_of(m, u), len = m.tb.clamped(m.len[u], m.status);
  constexpr int kRows = kShiftThreads / 4;
  for (int base = 0; base < n; base += kRows * kShiftUnroll) {
    uint4 x[kShiftUnroll];
    long long to[kShiftUnroll];
#pragma unroll
    for (int j = 0; j < kShiftUnroll; ++j) {
      const int i = base + j * kRows + r0;
      long long from;
      to[j] = -1;
      if (i < n && kept_row(m, idx, table, len, table, first, true, u, i, &from, &to[j]) &&
          from != to[j])
        x[j] = pool[from * kRow16 + ch];
      else
        to[j] = -1;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kShiftUnroll; ++j)
      if (to[j] >= 0) pool[to[j] * kRow16 + ch] = x[j];
    __syncthreads();
  }
}

int row16_of(const CacheShape& s) { return kD * (s.dtype == GRKV_F32 ? 4 : 2) / 16; }

// A launch of k_cache_fork or k_cache_trim, 1024 entries a block.  Up to 2 K entries go to one
// block, which also writes the status: its second round costs what a memset does (1.2 us).
template <typename... Params, typename... Args>
int table_call(const CacheShape& s, const CacheWs& L, char* ws, cudaStream_t st,
               void (*kern)(Params...), Args&&... args) {
  const int entries = s.U * s.cols;
  const bool solo = entries <= 1 << 11;
  if (!solo) GRKV_TRY(clear_status(ws, L, st));
  count_launches(1);
  return cuda_rc(launch_kernel(false, 1, kern, dim3(solo ? 1u : (unsigned)((entries + 1023) / 1024)), 1024,
                               0, st, table_of(s), std::forward<Args>(args)..., (int*)(ws + L.status),
                               solo));
}

// A launch of k_cache_append or k_cache_gather: rows of 16 (bf16) or 32 (fp32) chunks.
template <typename... Params, typename... Args>
cudaError_t launch_rows(const CacheShape& s, void (*k16)(Params...), void (*k32)(Params...),
                        cudaStream_t st, Args&&... args) {
  const int row16 = row16_of(s), rows = move_rows(row16);
  count_launches(1);
  return launch_kernel(false, 1, row16 == 16 ? k16 : k32,
                       dim3((unsigned)((s.t + rows - 1) / rows), (unsigned)std::min(s.U, 65535)),
                       kMoveThreads, 0, st, std::forward<Args>(args)...);
}

int attend(const grkv_cache_params* p, const AttendIo& io, bool tree, void* ws, size_t ws_bytes,
           void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (io.cross) s.W = 0;
  if ((tree && s.t > kMaxTree) || attend_tiles(s) > kMaxAttendTiles) return GRKV_ERR_UNSUPPORTED;
  cudaStream_t st = (cudaStream_t)stream;
  if (s.U == 0) return clear_status((char*)ws, L, st);
  GRKV_TRY(check_ptrs({io.q, io.k, io.v, io.out}, 16));
  GRKV_TRY(check_ptrs({io.table, io.len}, 4));
  if (tree) GRKV_TRY(check_ptrs({io.parent}, 4));
  GRKV_TRY(check_optional(io.qlen, 4));
  GRKV_TRY(check_optional(io.lse, 4));
  return cuda_rc(launch_attend(s, io, (char*)ws, L, st));
}

}  // namespace

cudaError_t grkv::launch_clear_status(int* word, cudaStream_t st) {
  count_launches(1);
  return launch_kernel(false, 1, k_clear_status, dim3(1), 1, 0, st, word);
}

extern "C" {

void grkv_cache_params_init(grkv_cache_params* p, int32_t units, int32_t group, int32_t pages,
                            int32_t page, int32_t max_pages) {
  if (!p) return;
  p->units = units;
  p->group = group;
  p->d = kD;
  p->pages = pages;
  p->page = page;
  p->max_pages = max_pages;
  p->tokens = 1;
  p->window = 0;
  p->n_sink = 4;
  p->scale = 0.f;
  p->dtype = GRKV_BF16;
  p->flags = 0;
}

int grkv_cache_workspace_size(const grkv_cache_params* p, size_t* bytes) {
  CacheShape s;
  GRKV_TRY(make_cache_shape(p, &s));
  if (!bytes) return GRKV_ERR_INVALID_ARG;
  *bytes = plan_cache_ws(s).total;
  return GRKV_OK;
}

int grkv_attend(const grkv_cache_params* p, const void* q, const void* k_pages, const void* v_pages,
                const int32_t* table, const int32_t* len, const int32_t* q_len, void* out,
                float* lse, void* ws, size_t ws_bytes, void* stream) {
  const AttendIo io{q, k_pages, v_pages, table, len, q_len, nullptr, out, lse, false};
  return attend(p, io, false, ws, ws_bytes, stream);
}

int grkv_attend_tree(const grkv_cache_params* p, const void* q, const void* k_pages,
                     const void* v_pages, const int32_t* table, const int32_t* len,
                     const int32_t* q_len, const int32_t* parent, void* out, float* lse, void* ws,
                     size_t ws_bytes, void* stream) {
  const AttendIo io{q, k_pages, v_pages, table, len, q_len, parent, out, lse, false};
  return attend(p, io, true, ws, ws_bytes, stream);
}

int grkv_attend_cross(const grkv_cache_params* p, const void* q, const void* k_pages,
                      const void* v_pages, const int32_t* table, const int32_t* len,
                      const int32_t* q_len, void* out, float* lse, void* ws, size_t ws_bytes,
                      void* stream) {
  const AttendIo io{q, k_pages, v_pages, table, len, q_len, nullptr, out, lse, true};
  return attend(p, io, false, ws, ws_bytes, stream);
}

int grkv_cache_fork(const grkv_cache_params* p, int32_t units_in, const int32_t* src,
                    const int32_t* table_in, const int32_t* len_in, int32_t* table_out,
                    int32_t* len_out, int32_t* refs, void* ws, size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (units_in < 0) return GRKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({src, table_out, len_out, refs}, 4));
    if (units_in > 0) GRKV_TRY(check_ptrs({table_in, len_in}, 4));
    if (table_in == table_out || len_in == len_out) return GRKV_ERR_INVALID_ARG;
  }
  if (s.U == 0) return clear_status((char*)ws, L, st);
  return table_call(s, L, (char*)ws, st, k_cache_fork, units_in, src, table_in, len_in, table_out,
                    len_out, refs);
}

int grkv_cache_trim(const grkv_cache_params* p, int32_t* table, const int32_t* len, int32_t* refs,
                    void* ws, size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (s.U > 0) GRKV_TRY(check_ptrs({table, len, refs}, 4));
  cudaStream_t st = (cudaStream_t)stream;
  if (s.U == 0) return clear_status((char*)ws, L, st);
  return table_call(s, L, (char*)ws, st, k_cache_trim, table, len, refs);
}

int grkv_cache_reserve(const grkv_cache_params* p, int32_t* table, const int32_t* len,
                       const int32_t* want, int32_t* refs, void* k_pages, void* v_pages, void* ws,
                       size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({k_pages, v_pages}, 16));
    GRKV_TRY(check_ptrs({table, len, want, refs}, 4));
  }
  cudaStream_t st = (cudaStream_t)stream;
  char* w = (char*)ws;
  if (s.U == 0) return clear_status(w, L, st);
  count_launches(2);
  GRKV_TRY(cuda_rc(launch_kernel(false, 1, k_cache_reserve, dim3(1), kReserveThreads, 0, st,
                                 table_of(s), table, len, want, refs, (int32_t*)(w + L.list),
                                 (int4*)(w + L.jobs), (int*)(w + L.status))));
  return cuda_rc(launch_kernel(true, 1, k_cache_copy, dim3(std::min(s.U, 65535)), 256, 0, st, s.U,
                               row16_of(s), s.page, (const int4*)(w + L.jobs), (uint4*)k_pages,
                               (uint4*)v_pages));
}

int grkv_cache_append(const grkv_cache_params* p, const void* k_new, const void* v_new,
                      const int64_t* first_row, int64_t new_rows, const int32_t* count,
                      const int32_t* table, const int32_t* len, void* k_pages, void* v_pages,
                      void* ws, size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({k_new, v_new, k_pages, v_pages}, 16));
    GRKV_TRY(check_ptrs({table, len}, 4));
  }
  GRKV_TRY(check_optional(first_row, 8));
  if (first_row && new_rows < 0) return GRKV_ERR_INVALID_ARG;
  GRKV_TRY(check_optional(count, 4));
  cudaStream_t st = (cudaStream_t)stream;
  GRKV_TRY(clear_status((char*)ws, L, st));
  if (s.U == 0) return GRKV_OK;
  const RowMove m{table_of(s), s.t, count, len, (int*)((char*)ws + L.status)};
  return cuda_rc(launch_rows(s, k_cache_append<16>, k_cache_append<32>, st, m, (const uint4*)k_new,
                             (const uint4*)v_new, first_row,
                             first_row ? (long long)new_rows : (long long)s.U * s.t, table, (uint4*)k_pages,
                             (uint4*)v_pages));
}

int grkv_cache_compact(const grkv_cache_params* p, const int32_t* idx, const int32_t* keep,
                       const int32_t* first, const int32_t* table_in, const int32_t* len_in,
                       const int32_t* table_out, void* k_pages, void* v_pages, void* ws,
                       size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({k_pages, v_pages}, 16));
    GRKV_TRY(check_ptrs({idx, table_in, len_in, table_out}, 4));
  }
  GRKV_TRY(check_optional(keep, 4));
  GRKV_TRY(check_optional(first, 4));
  cudaStream_t st = (cudaStream_t)stream;
  GRKV_TRY(clear_status((char*)ws, L, st));
  if (s.U == 0) return GRKV_OK;
  const RowMove m{table_of(s), s.t, keep, len_in, (int*)((char*)ws + L.status)};
  uint4 *k = (uint4*)k_pages, *v = (uint4*)v_pages;
  if (table_in != table_out)
    return cuda_rc(launch_rows(s, k_cache_gather<16>, k_cache_gather<32>, st, m, idx, table_in,
                               table_out, first, k, v));
  count_launches(1);
  const int row16 = row16_of(s);
  return cuda_rc(launch_kernel(false, 1, row16 == 16 ? k_cache_shift<16> : k_cache_shift<32>,
                               dim3(s.U, 2, row16 / 4), kShiftThreads, 0, st, m, idx, table_in, first, k, v));
}

}  // extern "C"
