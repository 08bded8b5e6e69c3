// Attention over the paged cache: what the portable and the tensor-core kernel share.
// The visible slots of a row, the work items, their split over the CTAs, and the
// partial results that k_attend_join adds up.
//
// A work item is one unit and a block of its tokens: `nq` row tiles of T tokens x g
// query heads, which read the same keys.  Its keys come in tiles of 128 slots: those
// that hold sinks, then those of the rows' windows.  The items' tiles in a row
// are cut into equal runs, one per CTA, whatever item they belong to: lengths that
// differ, causal triangles, few units with many keys and many units with few all
// leave every CTA the same work, and only the device needs to know the lengths.  A CTA
// that holds only part of an item's tiles leaves a partial (reference, sum, output).
#pragma once

#include "cache_args.cuh"
#include "sm100.cuh"

namespace grkv {

constexpr int kSlotTile = 128;   // slots per key tile

struct AttendRec {
  int u, qb, last, err;   // the split item that starts in this CTA (u < 0: none), its last CTA
};

struct AttendArgs {
  const void *q, *k, *v;
  const int32_t *table, *len, *qlen, *parent;
  void* out;
  float* lse;
  int U, g, t, P, shift, cols, W, s;
  int T;       // tokens of a row tile
  int nq;      // row tiles of an item
  int QB;      // items of a unit
  int rows;    // rows of an item, nq * T * g
  int extra;   // tiles' worth of work of an item besides its tiles
  int wide;    // there may be 2^30 of them or more
  float sl2;   // scale * log2(e)
  AttendRec* rec;
  float2* pml;
  float* po;
  int* status;
  int withhold;   // GRKV_TEST_TIMEOUT: CTA 0 withholds one arrive (tensor cores)
  static constexpr bool cross = false;
  static constexpr int tile = kSlotTile;
  __device__ int extra_of(long long) const { return extra; }   // of a call of so many tiles
  __device__ bool tree() const { return parent != nullptr; }
};

// Of attention over encoder states: every row sees the whole unit, whose slots end at the items' base;
// rows are none of them.  A type of its own, so that the kernels of the others stay as they are
// (asked at run time, chunks took 364 us for 360, windowed prefill 190 for 187).
struct CrossArgs : AttendArgs {
  static constexpr bool cross = true;
  __device__ bool tree() const { return false; }
};
// ... in slot tiles of 64 (grkv_cross_split.cu).
struct SplitArgs : CrossArgs {
  static constexpr int tile = 64;
  // where CTAs have one tile each, there is nothing to even out
  __device__ int extra_of(long long all) const { return all > gridDim.x ? extra : 0; }
};

// One item: tokens [tok0, tok0 + ntok) of unit u; the slots that its rows see are in
// [0, sink_end) and [lo, hi); its tile k is slot tile k < ns ? k : lo_tile + k - ns.
struct Item {
  int u, tok0, ntok, base, L;
  int sink_end, lo, hi, ns, lo_tile, nt;
  __device__ int tile(int k) const { return k < ns ? k : lo_tile + k - ns; }
  // Slots [a, b) hold one that some row of the item sees.
  __device__ bool wanted(int a, int b) const { return a < sink_end || (a < hi && b > lo); }
};

// Item qb of a unit whose length and tokens (clamped) are known.
template <typename A>
__device__ __forceinline__ Item make_item(const A& a, int u, int qb, int L, int T) {
  Item it;
  it.u = u;
  it.L = L;
  it.base = A::cross ? L : L - T;
  it.tok0 = qb * a.nq * a.T;
  it.ntok = max(0, min(T - it.tok0, a.nq * a.T));
  const int p0 = it.base + (a.tree() ? 0 : it.tok0);   // the first position of a row
  it.hi = A::cross ? L : max(0, it.base + it.tok0 + it.ntok);
  it.lo = !A::cross && a.W ? min(max(0, p0 - a.W + 1), it.hi) : 0;
  it.sink_end = !A::cross && a.W ? min(a.s, it.lo) : 0;
  it.lo_tile = it.lo / A::tile;
  it.ns = min((it.sink_end + A::tile - 1) / A::tile, it.lo_tile);
  it.nt = it.ns + (it.hi + A::tile - 1) / A::tile - it.lo_tile;
  if (it.ntok == 0) it.nt = 0;
  else if (it.nt < 1) it.nt = 1;   // rows that see nothing are written by a tile without slots
  return it;
}

__device__ __forceinline__ int unit_len(const AttendArgs& a, int u) {
  return min(max(__ldg(a.len + u), 0), a.cols << a.shift);
}
__device__ __forceinline__ int unit_tokens(const AttendArgs& a, int u) {
  return a.qlen ? min(max(__ldg(a.qlen + u), 0), a.t) : a.t;
}
template <typename A>
__device__ __forceinline__ Item make_item(const A& a, int u, int qb) {
  return make_item(a, u, qb, unit_len(a, u), unit_tokens(a, u));
}

// The slot tiles that every row of tokens [t0, t0 + n) of an item sees whole: those that end
// by the first row's last slot and are sinks or start in the last row's window (in a tree a
// node's depth is at most its index).
struct FullTiles {
  int end, sinks, window;
  template <typename A>
  __device__ FullTiles(const A& a, const Item& it, int t0, int n) {
    const bool window_on = !A::cross && a.W;
    end = max(0, A::cross || a.tree() ? it.base : it.base + t0 + 1) / kSlotTile;
    sinks = window_on ? a.s / kSlotTile : 0;
    window = window_on ? (max(0, it.base + t0 + n - a.W) + kSlotTile - 1) / kSlotTile : 0;
  }
  __device__ bool has(int tile) const { return tile < end && (tile < sinks || tile >= window); }
};

// Bits 0..n-1 (n clamped to 0..32).
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}
// Bit e: slot a + e is in [x, y).
__device__ __forceinline__ uint32_t range_bits(int a, int x, int y) {
  return low_bits(y - a) & ~low_bits(x - a);
}

// What one row sees: slots below end_s or in [lo, hi), and, in a tree, the drafted
// slots base + b whose bit b is set in anc.
struct RowVis {
  int end_s, lo, hi, base;
  const uint32_t* anc;   // kMaxTree bits, or null
  // Bit e: slot a + e (a a multiple of 32).
  __device__ uint32_t word(int a) const {
    uint32_t m = range_bits(a, 0, end_s) | range_bits(a, lo, hi);
    if (anc) {
      const int o = a - base, i = o >> 5, sh = o & 31;   // arithmetic shift: floor
      const uint32_t w0 = (unsigned)i < kMaxTree / 32 ? anc[i] : 0u;
      const uint32_t w1 = (unsigned)(i + 1) < kMaxTree / 32 ? anc[i + 1] : 0u;
      m |= __funnelshift_r(w0, w1, sh);
    }
    return m;
  }
};

// The slots that token i of the item's unit sees (live: the row exists), for a segment whose
// slots end before `end`.  In a tree the row's ancestor bits go to anc, 8 words that only
// this thread writes; a bad parent sets *err and counts as none.  The walk up the tree, a
// chain of dependent loads, is made only where a drafted slot or a window needs it.
template <typename A>
__device__ __forceinline__ RowVis row_vis(const A& a, const Item& it, int i, bool live,
                                          int end, uint32_t* anc, int* err) {
  RowVis r{0, 0, 0, it.base, nullptr};
  const bool walk = a.tree() && (a.W || end > it.base);
  if (walk) {
#pragma unroll
    for (int w = 0; w < kMaxTree / 32; ++w) anc[w] = 0;
    r.anc = anc;
  }
  if (!live) return r;
  int p = it.base + i;
  r.hi = p + 1;
  if (walk) {
    const int32_t* par = a.parent + (size_t)it.u * a.t;
    int depth = 0, w = i >> 5;
    uint32_t bits = 1u << (i & 31);
    for (int x = i;;) {
      const int y = __ldg(par + x);
      if (y < -1 || y >= x) *err = GRKV_ERR_INVALID_ARG;
      if (y < 0 || y >= x) break;
      x = y;
      ++depth;
      if (x >> 5 != w) {   // words are left downwards
        anc[w] = bits;
        w = x >> 5;
        bits = 0;
      }
      bits |= 1u << (x & 31);
    }
    anc[w] = bits;
    p = it.base + depth;
    if (a.W && depth >= a.W)   // the ancestor k steps up, at position p - k, may be out of the window
      for (int x = i, k = 0; k <= depth; ++k) {
        if (k >= a.W && p - k >= a.s) anc[x >> 5] &= ~(1u << (x & 31));
        x = __ldg(par + x);
      }
  }
  if (A::cross || a.tree()) r.hi = it.base;
  r.hi = max(r.hi, 0);
  // (CrossArgs::W is 0; with a constant here ptxas 13.0.88 finds no registers for k_attend_few<bf16, 8>)
  r.lo = a.W ? min(max(0, p - a.W + 1), r.hi) : 0;
  r.end_s = min(a.s, r.lo);
  return r;
}

// Where the CTAs' runs start.  Positions count an item's tiles and, in front of them, a.extra for
// the work that it brings by itself (its queries, its results); CTA c starts at
// q c + r c / G, with total = q G + r.
template <typename I>   // of positions: 32 bits where they all fit
struct Split {
  I total, q;
  int r, G;
  float inv;
  // Few instructions rather than divisions: at a kernel's start each is fetched from afar.
  __device__ Split(I all, int ctas) : total(all), G(ctas) {
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"((float)ctas));
    q = sizeof(I) == 8 ? all / ctas : (I)((float)all * inv);
    I left = all - q * ctas;
    for (; left < 0; left += ctas) --q;        // one step at most below 2^22 tiles, 257 at 2^30
    for (; left >= ctas; left -= ctas) ++q;
    r = (int)left;
  }
  // r c / G through fp32: r c + 1/2 over G is at least 1 / (2 G) > 2^-10 from a whole number, and
  // below 2^9, so that an error of a few 2^-23 of it does not reach one
  __device__ I start(int c) const { return q * c + (int)(((float)(r * c) + 0.5f) * inv); }
  __device__ int owner(I t) const {
    int c = min(G - 1, (int)((float)t * ((float)G / (float)total)));
    while (c > 0 && start(c) > t) --c;
    while (c + 1 < G && start(c + 1) <= t) ++c;
    return c;
  }
};

// A CTA's run: `left` tiles from tile `off` of item (u, qb) on.
struct Run {
  int u, qb, off, left;
};

struct PlanSmem {
  Run run;
  AttendRec rec;
  long long warp_sum[32], first, last;   // tiles in front of the run, and up to its end
  int warp_items[32];
  int err;
};

__device__ __forceinline__ int warp_total(int x) { return __reduce_add_sync(0xffffffffu, x); }
__device__ __forceinline__ long long warp_total(long long x) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

template <typename I, typename A>
__device__ __forceinline__ Run plan_run_of(const A& a, PlanSmem* ps, int n) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int items = a.U * a.QB;
  const int per = (items + n - 1) / n, i0 = min(items, tid * per), i1 = min(items, i0 + per);
  if (tid == 0) {
    ps->err = 0;
    ps->run = Run{0, 0, 0, 0};
    ps->rec = AttendRec{-1, 0, 0, 0};
    ps->first = ps->last = 0;
  }
  __syncthreads();
  const int first_u = i0 / a.QB, first_qb = i0 - first_u * a.QB;
  I mine = 0;
  int live = 0, nt0 = 0;   // items with rows; the first one's tiles
  for (int i = i0, u = first_u, qb = first_qb, L = 0, T = 0; i < i1; ++i) {
    if (i == i0 || qb == 0) {
      L = unit_len(a, u);
      T = unit_tokens(a, u);
      if (L != __ldg(a.len + u) || (a.qlen && T != __ldg(a.qlen + u))) ps->err = GRKV_ERR_INVALID_ARG;
    }
    const int nt = make_item(a, u, qb, L, T).nt;
    if (i == i0) nt0 = nt;
    mine += nt;
    live += nt > 0;
    if (++qb == a.QB) {
      qb = 0;
      ++u;
    }
  }
  I scan = mine;
  int scan_live = live;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const I x = __shfl_up_sync(0xffffffffu, scan, d);
    const int y = __shfl_up_sync(0xffffffffu, scan_live, d);
    if (lane >= d) {
      scan += x;
      scan_live += y;
    }
  }
  if (lane == 31) {
    ps->warp_sum[warp] = scan;
    ps->warp_items[warp] = scan_live;
  }
  __syncthreads();
  // tiles and items in front of this thread's items, and of all
  const I sum = lane < n / 32 ? (I)ps->warp_sum[lane] : 0;
  const int cnt = lane < n / 32 ? ps->warp_items[lane] : 0;
  const I all = warp_total(sum), tiles_before = warp_total(lane < warp ? sum : (I)0);
  const int all_live = warp_total(cnt), front = warp_total(lane < warp ? cnt : 0) + scan_live - live;
  I tiles = tiles_before + scan - mine;
  if (all > 0) {
    const I extra = a.extra_of(all);
    const Split<I> sp(all + extra * all_live, (int)min((I)gridDim.x, all));
    const int c = blockIdx.x;
    I at = tiles + extra * front;
    const I end = at + mine + extra * live;
    const I t0 = sp.start(c), t1 = sp.start(c + 1);
    // each end of the run is in the items of one thread
    const bool first = at <= t0 && t0 < end, last = at < t1 && t1 <= end;
    if (c < sp.G && (first || last)) {
      for (int i = i0, u = first_u, qb = first_qb; i < i1; ++i) {
        const int nt = i == i0 ? nt0 : make_item(a, u, qb).nt;
        if (nt > 0) {
          const I from = at + extra, to = from + nt;   // its tiles
          if (at <= t0 && t0 < to) {
            const int off = (int)max((I)0, t0 - from);
            ps->run = Run{u, qb, off, 0};
            ps->first = tiles + off;
          }
          if (at < t1 && t1 <= to) ps->last = tiles + max((I)0, t1 - from);
          if (t0 <= from && from < t1 && t1 < to) ps->rec = AttendRec{u, qb, sp.owner(to - 1), 0};
          at = to;
          tiles += nt;
          if (at >= t1) break;
        }
        if (++qb == a.QB) {
          qb = 0;
          ++u;
        }
      }
    }
  }
  __syncthreads();
  Run run = ps->run;
  run.left = (int)(ps->last - ps->first);
  return run;
}

// Every thread of the block takes part (n threads, a multiple of 32).  Returns the CTA's run
// (left == 0: none); ps->rec holds the split item that starts in it, ps->err any fault of
// the lengths.
template <typename A>
__device__ __forceinline__ Run plan_run(const A& a, PlanSmem* ps, int n) {
  return a.wide ? plan_run_of<long long>(a, ps, n) : plan_run_of<int>(a, ps, n);
}

// A CTA's segments in order: each is a run of tiles of one item.
template <typename A>
struct Segments {
  Item it;
  int qb, off, cnt, left, L, T;
  __device__ Segments(const A& a, const Run& r) : qb(r.qb), off(r.off), left(r.left) {
    it.u = r.u;
    if (left > 0) {
      unit(a);
      load(a);
    }
  }
  __device__ void unit(const AttendArgs& a) {
    L = unit_len(a, it.u);
    T = unit_tokens(a, it.u);
  }
  __device__ void load(const A& a) {
    it = make_item(a, it.u, qb, L, T);
    cnt = min(left, it.nt - off);
  }
  __device__ bool more() const { return left > 0; }
  __device__ bool whole() const { return off == 0 && cnt == it.nt; }
  __device__ int end() const { return (it.tile(off + cnt - 1) + 1) * A::tile; }
  __device__ int slot(int cta) const { return off == 0 ? 2 * cta + 1 : 2 * cta; }
  __device__ void next(const A& a) {
    left -= cnt;
    off = 0;
    if (left <= 0) return;
    do {   // items without rows are passed; left > 0 says that one with rows follows
      if (++qb == a.QB) {
        qb = 0;
        ++it.u;
        unit(a);
      }
      load(a);
    } while (it.nt == 0);
  }
};

// The page entry of table column c of unit u, and the page to read: an entry outside the
// pool sets *err and stands for page 0.
__device__ __forceinline__ int page_of(const AttendArgs& a, int u, int c, int* err) {
  const int e = __ldg(a.table + (size_t)u * a.cols + c);
  if ((unsigned)e < (unsigned)a.P) return e;
  *err = GRKV_ERR_INVALID_ARG;
  return 0;
}

// Row r of row tile w of an item: its head and token; false for rows that are padding.
__device__ __forceinline__ bool row_of(const AttendArgs& a, const Item& it, int w, int r, int* h,
                                       int* i) {
  *h = r / a.T;
  const int x = w * a.T + r - *h * a.T;
  *i = it.tok0 + x;
  return *h < a.g && x < it.ntok;
}

// Four columns (from 4 c4) of row r of a CTA's part.  Parts are stored a column group after the
// other, rows inside, so that the tensor-core kernel's threads, a row each, write (and
// k_attend_join's read) 16 bytes next to each other.
__device__ __forceinline__ float4* part4(const AttendArgs& a, int slot, int c4, int r) {
  return (float4*)a.po + ((size_t)slot * (kD / 4) + c4) * a.rows + r;
}

// A product q k as a logit in log2 units, and what a logit weighs against a reference, itself a logit.  Each step is
// rounded by itself: where a compiler fused them, the product would be exact and the reference not, 2^-25 of it
// apart, which for logits of 2^33 is more than an exponent holds.
__device__ __forceinline__ float logit_of(float product, float sl2) { return __fmul_rn(product, sl2); }
__device__ __forceinline__ float prob_of(float logit, float ref) { return sm100::fast_exp2(__fsub_rn(logit, ref)); }

// What a partial result with reference m weighs against reference M.
__device__ __forceinline__ float weight_of(float m, float M) {
  return m == -INFINITY ? 0.f : sm100::fast_exp2(m - M);
}

// ln of a row's sum of exponentials; -inf for a row that sees nothing.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

__device__ __forceinline__ void store_row4(float* p, float4 x) { *(float4*)p = x; }
__device__ __forceinline__ void store_row4(__nv_bfloat16* p, float4 x) {
  uint2 v;
  v.x = sm100::pack_bf16(x.x, x.y);
  v.y = sm100::pack_bf16(x.z, x.w);
  *(uint2*)p = v;
}

// Attention over encoder states for few rows and small caches (grkv_attend_cross.cu).
bool cross_is_few(const CacheShape& s, int sms);
cudaError_t launch_cross_few(const CacheShape& s, const AttendArgs& a, int sms, cudaStream_t st);

// ... in fp32 for more rows, on the tensor cores (grkv_cross_split.cu).
bool cross_is_split(const CacheShape& s);
void split_rows(const CacheShape& s, AttendArgs* a);
cudaError_t launch_cross_split(const AttendArgs& a, int G, cudaStream_t st);

cudaError_t launch_attend_tc(const CacheShape& s, const AttendArgs& a, bool cross, int G, cudaStream_t st);

}  // namespace grkv
