// Attention over the paged cache on the 5th-generation tensor cores (bf16).
//
// A row tile is up to 128 rows: T tokens x g query heads, so that the heads of a
// group share every key that is loaded.  One CTA per SM walks its run of (item, slot
// tile) pairs (attend_plan.cuh); an item is one row tile, or two where a unit has more
// than 128 rows.  Per slot tile of 128:
//   S = Q K^T (tcgen05, TMEM)  ->  P = exp2(S scale log2 e - ref)  ->  O += P V (P in TMEM)
//
// Roles.  Warp 0 copies pages to a ring of 128-slot tiles by TMA, a box per page and
// half row (pages of 16 to 128 slots), and the items' queries.  Warp 1 issues the MMAs,
// the S product two jobs ahead of the P V product, so that the tensor cores work
// on one row tile (two-tile items) or one slot tile (one-tile items) while the softmax
// works on the other.  Warps 4-7 (and 8-11 for the second row tile) do the softmax: a
// thread owns one row, one TMEM lane, and holds the tile's 128 logits in registers.
// Warps 2-3 search the V of masked tiles (below).
//
// The reference of a row is the maximum of the first tile in which it sees a slot, and stays:
// P, O and the sum are floating point, so what counts is only that nothing leaves their
// range.  The first tile's largest P is 1, so no sum underflows; and where a later tile takes a row's
// sum past 2^60 the row takes that tile's maximum, the tile is done again and the output
// scaled in TMEM.  A running maximum costs 64 three-operand maxima per row and tile in front of
// the exponentials (half their time), and now and then the output's rescaling.
// The exponents come from one fused logit x scale - reference, in which the product is exact and the
// reference rounded: from 2^23 on by more than 1/2, and in the end by more than an exponent
// holds.  A row with such a reference follows the running maximum, rounded down, and its exponents are
// bounded by 0: logits that fp32 cannot tell from the maximum weigh as much as it.  That is done to the
// logits in TMEM, by code that such rows alone reach: in line it cost windowed trees and
// prompts 2%.  The tests and the sum over the whole run cost the chunk below 328 -> 334 us.
//
// P is rounded to bf16 for the product with V: a relative 2^-8 a term at most, of the size of
// the output's own rounding.  A row's sum is taken in fp32 before that.  A second product with
// what the rounding left, 512 cycles and the packing, is made where it is nearly free: in the first
// slot tile of a segment (with a cache's sinks, if that is where a unit starts) of items of up to
// 64 rows, which wait for memory: one query over 64 units of up to 16384 slots took 59 us
// against 57 (for every tile 65; 256 units of 32768: 680 against 624).  Items of more rows wait for the
// MMAs and the softmax and round once: trees of 65 rows over 128 units took 43.7 us against
// 45.5.  So a row's error depends on how many rows its call has a unit, and on where the split over
// the CTAs falls: 0.0017 (both parts, the size of the output's rounding) to 0.0020 of the outputs' size, within
// 2^-8 of sum p |v| in every case.
//
// What bounds it (one GB300).  Few rows over a long cache: memory, 256 units of 32768 slots in
// 625 us, 6.9 TB/s.  Chunks of prefill: a row tile's chain of S (512 cycles), softmax (1.2 K with two
// warps to a scheduler) and P V (512), which two row tiles overlap: 3.0 K cycles a slot tile against
// 2 K of MMAs; 2048 queries of 32 heads over 16384 slots take 334 us, 1.54 PFLOP/s, at 2070 MHz, and 357 us
// call after call for a second and more, when the power limit holds the clock at 1.94 to 1.97 GHz.  Windows
// and trees: items are short, and each has a start and an end (8 K cycles) and tiles with masks (2 K more).
//
// Slot tiles that every row sees whole take no masks.  In the others the masks of a row are
// four words, and V is searched for non-finite elements first: they are set to zero
// in shared memory (0 x NaN would reach rows that do not see the slot; what was
// never loaded is there too) and added again, at the end, to the rows that do see them.
#include <stddef.h>

#include <algorithm>
#include <type_traits>

#include "attend_plan.cuh"
#include "tmap.cuh"

namespace grkv {
namespace {

using namespace sm100;

constexpr int kRows = 128;                                    // rows of a tile, TMEM lanes
constexpr uint32_t kTileBytes = kSlotTile * kD * 2;           // 32 KB
constexpr int kRing = 4;   // tiles in flight: K in the even slots, V in the odd ones
constexpr long long kWaitBudget = 1ll << 32;                  // cycles (~2 s)
constexpr long long kTestWaitBudget = 1ll << 22;              // ~2 ms: GRKV_TEST_TIMEOUT's
constexpr int kMaxEdges = 16;   // masked tiles of a segment: at most 4 at each end of the
                                // window (256 tokens) and one at the sinks' end
constexpr float kMaxSum = 0x1p60f;   // of a row's P over a segment (a NaN stays as it is)
constexpr float kBigRef = 0x1p23f;   // references from here on are rounded by more than 1/2
constexpr int kFewRows = 64;   // up to which P keeps its low part in a segment's first tile
constexpr uint32_t kColO = 256; // TMEM: two S buffers, then two outputs

template <int NQ>
struct TcLayout {
  static constexpr int kQBufs = NQ == 1 ? 2 : 1;
  static constexpr int kThreads = 128 + NQ * 128;
  static constexpr uint32_t kOffQ = 0;
  static constexpr uint32_t kOffRing = 2 * kTileBytes;
  static constexpr uint32_t kOffAnc = kOffRing + kRing * kTileBytes;
  static constexpr uint32_t kOffBad = kOffAnc + NQ * kRows * (kMaxTree / 8);
  static constexpr uint32_t kOffBar = kOffBad + 4 * kMaxEdges * 16;
  static constexpr uint32_t kOffPlan = kOffBar + 512;
  static constexpr uint32_t kOffStage = kOffPlan + 1024;   // 2 KB a softmax warp
  static constexpr uint32_t kBytes = kOffStage + NQ * 4 * 2048 + 1024;   // + alignment slack
};
static_assert(TcLayout<2>::kBytes <= 227 * 1024 && sizeof(PlanSmem) <= 1024, "smem");

// Arrivals that complete a phase: 4 softmax warps, 2 searchers, else one.
struct TcBars {
  uint64_t p_full[2];     // 4: P written
  uint64_t v_ok[2];       // 2: V of the slot has been passed by both searchers
  uint64_t searched[4];   // 2: V of a masked tile has been searched (uses in turn)
  uint64_t ring_full[kRing], ring_empty[kRing], q_full[2], q_empty[2], s_full[2], o_done[2], drain;
  uint32_t tmem;
  int abort;
};
constexpr int kBars = 8 + 2 * kRing + 9;
static_assert(sizeof(TcBars) <= 512 && kBars <= 32 && offsetof(TcBars, tmem) == 8 * kBars, "barriers");

struct Ring {
  uint32_t slot = 0, phase = 0;
  __device__ void add(uint32_t k) {
    slot += k;
    if (slot >= kRing) {
      slot -= kRing;
      phase ^= 1;
    }
  }
};

// With two row tiles the softmax threads, which hold 128 logits each, get registers of the
// other warpgroup: 128 x 72 + 256 x 208 = 62464 of the 384 x 168 = 64512 at launch.
template <int NQ>
__device__ __forceinline__ void fewer_regs() {
  if (NQ == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
}
template <int NQ>
__device__ __forceinline__ void more_regs() {
  if (NQ == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
}

__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort,
                                          long long budget = kWaitBudget) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, budget));
}
__device__ __forceinline__ void arrive_warp(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ float max32(const float* v) {
  float m[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    m[c] = max3(v[c], v[4 + c], v[8 + c]);
    m[c] = max3(m[c], v[12 + c], v[16 + c]);
    m[c] = max3(m[c], v[20 + c], v[24 + c]);
    m[c] = fmaxf(m[c], v[28 + c]);
  }
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// exp2(v sl2 - r) of 32 logits as 16 bf16 pairs, and with kLow 16 more of what that rounding
// leaves; the sums are of the values before rounding.
template <bool kLow>
__device__ __forceinline__ void exp32(const float* v, float sl2, float r, uint32_t* pk, uint64_t* acc) {
  const uint64_t s2 = pack2(sl2, sl2), m2 = pack2(-r, -r);
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    float p0, p1;
    unpack2(fma2(pack2(v[2 * x], v[2 * x + 1]), s2, m2), p0, p1);
    p0 = fast_exp2(p0);
    p1 = fast_exp2(p1);
    acc[x & 3] = add2(acc[x & 3], pack2(p0, p1));
    pk[x] = pack_bf16(p0, p1);
    if (kLow)
      pk[16 + x] = pack_bf16(p0 - __uint_as_float(pk[x] << 16), p1 - __uint_as_float(pk[x] & 0xffff0000u));
  }
}

// Where some row of the warp has a large reference: every row takes the maximum `top`, and the logits
// of those with large ones become their exponents, bounded by 0, over the scale, so that the code that
// follows takes them against 0; a NaN stays (all lanes of the warp; rare, so not in line).
struct Followed {
  float ref, f;   // the new reference; what the row's output so far is multiplied by
};
__device__ __noinline__ Followed follow_row(uint32_t s_addr, float sl2, float top, float ref) {
  float to = top * sl2;
  if (!(fabsf(to) < kBigRef)) to = __fmul_rd(top, sl2);
  to = fmaxf(ref, to);
  const bool big = to != -INFINITY && !(fabsf(to) < kBigRef);
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    float v[32];
    tmem_ld32f(s_addr + 32 * c, v);
    tmem_wait32(v);
#pragma unroll
    for (int x = 0; x < 32; ++x) {
      const float t = fmaf(v[x], sl2, -to);
      if (big) v[x] = (t > 0.f ? 0.f : t) / sl2;
    }
    tmem_st16(s_addr + 32 * c, (uint32_t*)v);
    tmem_st16(s_addr + 32 * c + 16, (uint32_t*)v + 16);
  }
  tmem_st_wait();
  return Followed{to, ref == -INFINITY ? 1.f : fast_exp2(ref - to)};
}

// What the exponents are taken against: 0 for a row without a reference or with a large one.
__device__ __forceinline__ float against(float ref) { return fabsf(ref) < kBigRef ? ref : 0.f; }

// Multiplies a row's output by f (all lanes of the warp; rare, so not in line).
__device__ __noinline__ void scale_row(uint32_t o_addr, float f) {
  tc_fence_after();
  for (int c = 0; c < kD; c += 32) {
    float o[32];
    tmem_ld32f(o_addr + c, o);
    tmem_wait32(o);
#pragma unroll
    for (int x = 0; x < 32; ++x) o[x] *= f;
    tmem_st16(o_addr + c, (uint32_t*)o);
    tmem_st16(o_addr + c + 16, (uint32_t*)o + 16);
  }
  tmem_st_wait();
}

// Stores 64 bytes of each of a warp's 32 rows, x this lane's, through shared memory so that four
// lanes write a row's 64 bytes together (a lane to a row, every store touches 32 lines:
// an item's end took 8 K cycles of the load-store unit).  rows[j] is the index of row
// 8 j + lane / 4 in the array at base, or negative.
__device__ __forceinline__ void store_rows(uint8_t* stage, int lane, const uint4* x, const int* rows,
                                           uint8_t* base, size_t row_bytes) {
#pragma unroll
  for (int c = 0; c < 4; ++c) *(uint4*)(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = x[c];
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 8 * j + (lane >> 2), c = lane & 3;
    const uint4 y = *(const uint4*)(stage + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
    if (rows[j] >= 0) *(uint4*)(base + (size_t)rows[j] * row_bytes + c * 16) = y;
  }
  __syncwarp();
}

__device__ __forceinline__ bool nonfinite16(uint32_t h) { return (h & 0x7f80u) == 0x7f80u; }

// Searches one row of a V tile (two 128-byte halves) for non-finite elements and zeroes
// them.  x 0 + sum stays zero over finite elements and NaN from the first other one on.
__device__ __forceinline__ bool clean_row(uint8_t* tile, int row) {
  uint32_t sum = 0;
#pragma unroll
  for (int c0 = 0; c0 < 16; ++c0) {
    const int c = ((c0 & 7) + row) & 7;   // lanes on different banks
    const uint4 x = *(const uint4*)(tile + (c0 >> 3) * (kTileBytes / 2) + row * 128 + c * 16);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(w[i]), "r"(0u));
  }
  if (!nonfinite16(sum) && !nonfinite16(sum >> 16)) return false;
  for (int c = 0; c < 64; ++c) {
    uint32_t* w = (uint32_t*)(tile + (c >> 5) * (kTileBytes / 2) + row * 128) + (c & 31);
    uint32_t x = *w;
    if (nonfinite16(x)) x &= 0xffff0000u;
    if (nonfinite16(x >> 16)) x &= 0x0000ffffu;
    *w = x;
  }
  return true;
}

// Adds the non-finite values of the slots that a row sees to its output in TMEM (all lanes of the
// warp).  A function of its own: the epilogue's registers stay registers.
template <typename A>
__device__ __noinline__ void add_bad(const A& a, const Item& it, int off, int cnt,
                                     const RowVis& vis, const uint4* bad, bool live, uint32_t taddr) {
  int err = 0;
  for (int c0 = 0; c0 < kD; c0 += 32) {
    float o[32];
    tmem_ld32f(taddr + c0, o);
    tmem_wait32(o);
    int e = 0;
    const FullTiles full(a, it, it.tok0, it.ntok);
    for (int k = 0; live && k < cnt; ++k) {
      const int tile = it.tile(off + k);
      if (full.has(tile)) continue;
      const uint4 words = bad[min(e, kMaxEdges - 1)];
      const uint32_t w[4] = {words.x, words.y, words.z, words.w};
      ++e;
      for (int i = 0; i < 4; ++i) {
        const int x = tile * kSlotTile + 32 * i;
        for (uint32_t m = w[i] & vis.word(x); m; m &= m - 1) {
          const int slot = x + __ffs(m) - 1, c = slot >> a.shift;
          const size_t row =
              ((size_t)page_of(a, it.u, c, &err) << a.shift) + (slot & ((1 << a.shift) - 1));
          const __nv_bfloat16* v = (const __nv_bfloat16*)a.v + row * kD + c0;
          for (int j = 0; j < 32; ++j) {
            const float y = __bfloat162float(v[j]);
            if (!isfinite(y)) o[j] += y;
          }
        }
      }
    }
    __syncwarp();
    tmem_st16(taddr + c0, (uint32_t*)o);
    tmem_st16(taddr + c0 + 16, (uint32_t*)o + 16);
  }
  tmem_st_wait();
}

template <int NQ, typename A>
__global__ void __launch_bounds__(TcLayout<NQ>::kThreads, 1)
    k_attend_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                const __grid_constant__ CUtensorMap tmV, const __grid_constant__ A a) {
  using Lay = TcLayout<NQ>;
  extern __shared__ __align__(1024) uint8_t smraw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
  TcBars* bars = (TcBars*)(sm + Lay::kOffBar);
  PlanSmem* plan = (PlanSmem*)(sm + Lay::kOffPlan);
  uint4* bad_all = (uint4*)(sm + Lay::kOffBad);   // [4][kMaxEdges]
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // warp-uniform for the compiler

  if (warp == 0) {   // a barrier a lane: the instructions of a start are fetched one by one
    if (lane < kBars) mbar_init((uint64_t*)bars + lane, lane < 2 ? 4 : lane < 8 ? 2 : 1);
    if (lane == 0) {
      bars->abort = 0;
      prefetch_tensormap(&tmQ);
      prefetch_tensormap(&tmK);
      prefetch_tensormap(&tmV);
    }
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  const Run run = plan_run(a, plan, Lay::kThreads);   // ends with a barrier
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  volatile int* abort_flag = &bars->abort;
  int err = 0;
  const bool few = NQ == 1 && a.rows <= kFewRows;   // the first slot tile takes both parts of P

  if (warp == 0) {
    // -------------------------------------------------------------- producer
    fewer_regs<NQ>();
    const uint64_t keep = l2_evict_normal();
    const int per_tile = kSlotTile >> a.shift;
    const uint32_t page_bytes = 128u << a.shift;   // of one half
    uint32_t issued = 0;
    int seg = 0;
    Ring pos;
    bool ok = true;
    for (Segments<A> sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
      const Item& it = sg.it;
      const int qb = seg % Lay::kQBufs, quse = seg / Lay::kQBufs;
      if (quse >= 1) ok = wait_warp(&bars->q_empty[qb], (quse - 1) & 1, abort_flag);
      if (!ok) break;
      if (lane == 0) {
        mbar_expect_tx(&bars->q_full[qb], NQ * 256u * a.T * a.g);
#pragma unroll
        for (int w = 0; w < NQ; ++w) {
          uint8_t* dst = sm + Lay::kOffQ + (qb * NQ + w) * kTileBytes;
          const int i = it.tok0 + w * a.T;   // tokens past the last read as zeros
          tma_load_3d(dst, &tmQ, &bars->q_full[qb], 0, i, it.u * a.g, keep);
          tma_load_3d(dst + kTileBytes / 2, &tmQ, &bars->q_full[qb], 64, i, it.u * a.g, keep);
        }
      }
      // the page of this lane in tile k of the segment, or -1; the next tile's is asked for before
      // this one's slots are waited for
      auto look_up = [&](int k, bool* has) {
        const int c = it.tile(sg.off + k) * per_tile + lane;
        *has = lane < per_tile && c < a.cols && it.wanted(c << a.shift, (c + 1) << a.shift);
        return *has ? __ldg(a.table + (size_t)it.u * a.cols + c) : 0;
      };
      bool has, mine;
      int entry = look_up(0, &has);
      for (int k = 0; ok && k < sg.cnt; ++k) {
        mine = has;
        int page = entry;
        if (k + 1 < sg.cnt) entry = look_up(k + 1, &has);
        if (mine && (unsigned)page >= (unsigned)a.P) {   // an entry outside the pool: page 0
          err = GRKV_ERR_INVALID_ARG;
          page = 0;
        }
        const uint32_t n = __popc(__ballot_sync(0xffffffffu, mine));
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          if (issued >= kRing) ok = wait_warp(&bars->ring_empty[pos.slot], pos.phase ^ 1, abort_flag);
          if (!ok) break;
          uint64_t* full = &bars->ring_full[pos.slot];
          if (lane == 0) mbar_expect_tx(full, n * 2 * page_bytes);
          __syncwarp();
          if (mine) {
            uint8_t* dst = sm + Lay::kOffRing + pos.slot * kTileBytes + lane * page_bytes;
            const CUtensorMap* map = which ? &tmV : &tmK;
            tma_load_3d(dst, map, full, 0, 0, page, keep);
            tma_load_3d(dst + kTileBytes / 2, map, full, 64, 0, page, keep);
          }
          ++issued;
          pos.add(1);
        }
      }
    }
    // every issued load lands before the CTA can exit (these waits ignore the abort flag)
    volatile int no_abort = 0;
    for (uint32_t i = issued > kRing ? issued - kRing : 0; i < issued; ++i)
      mbar_wait(&bars->ring_full[i % kRing], (i / kRing) & 1, &no_abort, kWaitBudget);
    for (int s = max(0, seg - Lay::kQBufs); s < seg; ++s)
      mbar_wait(&bars->q_full[s % Lay::kQBufs], (s / Lay::kQBufs) & 1, &no_abort, kWaitBudget);
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------- MMA issuer
    // One warp feeds the tensor cores through some forty dependent instructions a product; with
    // the masks' tests and general ring positions in it, it was what bound the kernel (3.7 K
    // cycles for two row tiles of 2 K cycles of MMAs).  So tiles go two to a round: slots and
    // S buffers are constants, parities one bit; a segment only shows where its count ends.
    fewer_regs<NQ>();
    constexpr uint32_t id_s = idesc_bf16(kRows, kSlotTile, 0, 0);   // S = Q K^T, both K-major
    constexpr uint32_t id_o = idesc_bf16(kRows, kD, 0, 1);          // O += P V, V MN-major
    constexpr uint32_t kTileDesc = kTileBytes >> 4;
    const uint64_t q_desc = sw128_desc(smem_u32(sm + Lay::kOffQ), 16, 1024);
    const uint64_t k_desc = sw128_desc(smem_u32(sm + Lay::kOffRing), 16, 1024);
    const uint64_t v_desc = sw128_desc(smem_u32(sm + Lay::kOffRing + kTileBytes), kTileBytes / 2, 1024);
    auto wait = [&](uint64_t* bar, uint32_t parity) { return wait_warp(bar, parity, abort_flag); };
    // segments: the S products' (ahead), and the lengths of those the output's have yet to start
    Segments<A> qs(a, run);
    int q_left = 0, q_seg = -1, v_left = 0, v_seg = -1, next1 = 0, next2 = 0;
    uint32_t qb = 0;
    bool v_first = false;
    auto q_begin = [&]() -> bool {   // before a slot tile's S products
      if (q_left > 0) return true;
      if (q_seg >= 0) qs.next(a);
      ++q_seg;
      q_left = qs.cnt;
      if (next1 == 0) next1 = q_left;
      else next2 = q_left;
      qb = q_seg % Lay::kQBufs;
      return wait(&bars->q_full[qb], (q_seg / Lay::kQBufs) & 1);
    };
    auto q_end = [&]() {
      if (--q_left == 0) mma_commit_elect(&bars->q_empty[qb]);
    };
    auto v_begin = [&]() {   // before a slot tile's output products
      v_first = v_left == 0;
      if (v_first) {
        ++v_seg;
        v_left = next1;
        next1 = next2;
        next2 = 0;
      }
      --v_left;
    };
    auto issue_s = [&](int buf, int w, int slot) {
      mma8_ss<id_s>(tmem + buf * kSlotTile, q_desc + (qb * NQ + w) * kTileDesc,
                    k_desc + slot * 2 * kTileDesc);
    };
    auto issue_o = [&](int buf, int o, int slot) {
      tc_fence_after();
      const uint32_t d = tmem + kColO + o * kD, p = tmem + buf * kSlotTile;
      const uint64_t v = v_desc + slot * 2 * kTileDesc;
      mma8_ts<id_o, false>(d, p, v, !v_first);
      if (few && v_first) mma8_ts<id_o, false>(d, p + 16, v, true);   // what the rounding of P left
    };
    const int tiles = run.left;
    // Slot tile t, in slot B = t & 1; ph = (t >> 1) & 1.  With two row tiles everything but P is
    // waited for first, so that nothing stands between a product with V and the S product
    // over its P, and one signal says that both are done; the output's own is for a
    // segment's end.  One row tile is bound by memory: V is given back as early as can be.
    auto step = [&](auto b_const, int t, uint32_t ph) -> bool {
      constexpr int B = decltype(b_const)::value;
      v_begin();
      if (!wait(&bars->v_ok[B], ph)) return false;
      if (NQ == 2) {
        const bool more = t + 1 < tiles;
        auto k_ready = [&]() { return wait(&bars->ring_full[2 * (1 - B)], B ? ph ^ 1 : ph); };
        auto s_done = [&]() {
          mma_commit_elect(&bars->s_full[1]);
          mma_commit_elect(&bars->ring_empty[2 * (1 - B)]);
          q_end();
        };
        if (more && q_left > 0) {
          if (!k_ready() || !wait(&bars->p_full[0], B)) return false;
          issue_o(0, 0, B);
          issue_s(0, 0, 1 - B);
          mma_commit_elect(&bars->s_full[0]);
          if (!wait(&bars->p_full[1], B)) return false;
          issue_o(1, 1, B);
          issue_s(1, NQ - 1, 1 - B);
          s_done();
        } else {   // the segment's last tile: its outputs do not wait for the next one's queries
          if (!wait(&bars->p_full[0], B)) return false;
          issue_o(0, 0, B);
          mma_commit_elect(&bars->o_done[0]);
          if (!wait(&bars->p_full[1], B)) return false;
          issue_o(1, 1, B);
          mma_commit_elect(&bars->o_done[1]);
          if (more) {
            if (!q_begin() || !k_ready()) return false;
            issue_s(0, 0, 1 - B);
            mma_commit_elect(&bars->s_full[0]);
            issue_s(1, NQ - 1, 1 - B);
            s_done();
          }
        }
        mma_commit_elect(&bars->ring_empty[2 * B + 1]);
      } else {
        if (!wait(&bars->p_full[B], ph)) return false;
        issue_o(B, v_seg & 1, B);
        mma_commit_elect(&bars->o_done[B]);
        mma_commit_elect(&bars->ring_empty[2 * B + 1]);
        if (t + 2 < tiles) {   // K of tile t + 2 may still be on its way from memory
          if (!q_begin() || !wait(&bars->ring_full[2 * B], ph ^ 1)) return false;
          issue_s(B, 0, B);
          mma_commit_elect(&bars->s_full[B]);
          mma_commit_elect(&bars->ring_empty[2 * B]);
          q_end();
        }
      }
      return true;
    };
    bool ok = true;
    for (int t = 0; t < (NQ == 2 ? 1 : 2) && t < tiles && ok; ++t) {   // the first S products
      ok = q_begin() && wait(&bars->ring_full[2 * t], 0);
      if (!ok) break;
      issue_s(t, 0, t);
      mma_commit_elect(&bars->s_full[t]);
      if (NQ == 2) {
        issue_s(1, NQ - 1, t);
        mma_commit_elect(&bars->s_full[1]);
      }
      mma_commit_elect(&bars->ring_empty[2 * t]);
      q_end();
    }
    for (int t = 0; ok && t < tiles; t += 2) {
      const uint32_t ph = (t >> 1) & 1;
      ok = step(std::integral_constant<int, 0>{}, t, ph);
      if (ok && t + 1 < tiles) ok = step(std::integral_constant<int, 1>{}, t + 1, ph);
    }
    // every MMA issued so far completes before TMEM is released
    mma_commit_elect(&bars->drain);
    volatile int no_abort = 0;
    mbar_wait(&bars->drain, 0, &no_abort, kWaitBudget);
    __syncwarp();
  } else if (warp < 4) {
    // --------------------------------------------------- search of masked tiles' V
    fewer_regs<NQ>();
    // Two warps, two rows a lane.  They pass every V tile in turn, masked or not, and its product
    // waits for them: so a parity always means the use that they are at, and they are ahead
    // of the softmax by at most the ring's two V tiles, which four marks and four segments'
    // words cover.
    uint32_t edges = 0;
    int seg = 0;
    Ring vp;
    vp.add(1);
    // GRKV_TEST_TIMEOUT: one warp of CTA 0 never says that it has passed the first V tile, so that
    // nothing goes on, and is the first to give up
    bool withhold = a.withhold && blockIdx.x == 0 && warp == 2;
    const long long budget = withhold ? kTestWaitBudget : kWaitBudget;
    auto passed = [&]() {
      if (lane == 0 && !withhold) mbar_arrive(&bars->v_ok[vp.slot >> 1]);
      withhold = false;
    };
    bool ok = true;
    for (Segments<A> sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
      const Item& it = sg.it;
      const FullTiles full(a, it, it.tok0, it.ntok);
      int e = 0;
      for (int k = 0; ok && k < sg.cnt; ++k, vp.add(2)) {
        ok = wait_warp(&bars->ring_full[vp.slot], vp.phase, abort_flag, budget);
        if (!ok) break;
        if (full.has(it.tile(sg.off + k))) {
          passed();
          continue;
        }
        uint8_t* tile = sm + Lay::kOffRing + vp.slot * kTileBytes;
        uint32_t* words = (uint32_t*)(bad_all + (seg & 3) * kMaxEdges + e);
#pragma unroll 1
        for (int r = 0; r < 2; ++r) {
          const int q = (warp - 2) * 2 + r;
          // (what lies in slots that were not loaded may look like anything; no row sees it)
          const int slot = it.tile(sg.off + k) * kSlotTile + q * 32 + lane;
          const bool found = clean_row(tile, q * 32 + lane);
          const uint32_t bits = __ballot_sync(0xffffffffu, found && it.wanted(slot, slot + 1));
          if (lane == 0 && e < kMaxEdges) words[q] = bits;
          fence_proxy_async_smem();
        }
        arrive_warp(&bars->searched[edges & 3], lane);
        passed();
        ++edges;
        ++e;
      }
    }
  } else {
    // ---------------------------------------------------------------- softmax
    more_regs<NQ>();
    const int w = (warp - 4) >> 2, q = warp & 3, row = q * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(q * 32) << 16);
    uint32_t* anc = (uint32_t*)(sm + Lay::kOffAnc) + (w * kRows + row) * (kMaxTree / 32);
    uint32_t n = w, edges = 0;
    int seg = 0;
    bool ok = true;
    for (Segments<A> sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
      const Item& it = sg.it;
      int h, i;
      const bool live = row_of(a, it, w, row, &h, &i);
      const bool warp_live = __any_sync(0xffffffffu, live);
      const RowVis vis = row_vis(a, it, i, live, sg.end(), anc, &err);
      const int t0 = it.tok0 + w * a.T, nt = min(a.T, it.tok0 + it.ntok - t0);
      const FullTiles all_full(a, it, it.tok0, it.ntok), full(a, it, t0, nt);
      uint4* bad = bad_all + (seg & 3) * kMaxEdges;
      float ref = -INFINITY, l = 0.f;
      int e = 0;
      bool any_bad = false, follow = warp_live;   // some row has no reference yet, or a large one
      const uint32_t ocol = kColO + (NQ == 2 ? w : seg & 1) * kD;
      // The products of all tiles up to job `job` are in the output.  Two row tiles: S of job n has
      // been signalled after them, so only a segment's end has to wait, for its own signal.
      auto done = [&](uint32_t job, bool end) {
        if (NQ == 1) return wait_warp(&bars->o_done[job & 1], (job >> 1) & 1, abort_flag);
        return !end || wait_warp(&bars->o_done[w], seg & 1, abort_flag);
      };
      for (int k = 0; k < sg.cnt; ++k, n += NQ) {
        const int tile = it.tile(sg.off + k);
        const bool edge = !all_full.has(tile);
        const uint32_t scol = (n & 1) * kSlotTile;
        ok = wait_warp(&bars->s_full[n & 1], (n >> 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (warp_live) {
          const bool masked = !full.has(tile);
          float sum = 0.f, f = 1.f;
          bool look = follow;   // or a sum that left its range
          if (masked) {
            // -inf, in TMEM, for the slots that a row does not see: one chunk's code, for the
            // chunks that some row of the warp does not see whole.  (In line with the
            // exponentials, 128 selects more to fetch: the chunk above took 350 us where it took 329.)
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              const uint32_t m = vis.word(tile * kSlotTile + 32 * c);
              if (__all_sync(0xffffffffu, m == 0xffffffffu)) continue;
              float v[32];
              tmem_ld32f(lane_addr + scol + 32 * c, v);
              tmem_wait32(v);
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!((m >> x) & 1)) v[x] = -INFINITY;
              tmem_st16(lane_addr + scol + 32 * c, (uint32_t*)v);
              tmem_st16(lane_addr + scol + 32 * c + 16, (uint32_t*)v + 16);
            }
            tmem_st_wait();
          }
          // Such rows take the maximum; true: some reference is large, the logits have been changed.
          auto new_ref = [&](float top) -> bool {
            const bool need = live && (ref == -INFINITY || sum + l >= kMaxSum);
            const float before = ref, to = fmaxf(ref, top * a.sl2);
            if (need && ref != -INFINITY) f = fast_exp2(ref - to);
            if (need) ref = to;
            follow = __any_sync(0xffffffffu, live && !(fabsf(ref) < kBigRef));
            if (!follow || !__any_sync(0xffffffffu, live && ref != -INFINITY && !(fabsf(ref) < kBigRef)))
              return false;
            const Followed y = follow_row(lane_addr + scol, a.sl2, top, before);
            ref = y.ref;
            f = y.f;
            return true;
          };
          auto total = [&](const uint64_t* acc) {
            float s0, s1;
            unpack2(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), s0, s1);
            return s0 + s1;
          };
          if (few && k == 0) {
            // both parts of P; a chunk at a time, over the logits that it comes from
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {   // the maximum first
              float v[32];
              tmem_ld32f(lane_addr + scol + 32 * (c & 3), v);
              tmem_wait32(v);
              if (c < 4) {
                top = fmaxf(top, max32(v));
                if (c == 3) new_ref(top);
                continue;
              }
              uint32_t pk[32];
              uint64_t acc[4] = {0, 0, 0, 0};
              exp32<true>(v, a.sl2, against(ref), pk, acc);
              sum += total(acc);
              tmem_st16(lane_addr + scol + 32 * (c & 3), pk);
              tmem_st16(lane_addr + scol + 32 * (c & 3) + 16, pk + 16);
            }
          } else {
            uint32_t pk[64];
#pragma unroll 1
            for (bool again = false;; again = true) {
              // the first chunk's exponentials run while the others are on their way
              float v[128];
              tmem_ld32f(lane_addr + scol, v);
              tmem_wait32(v);
#pragma unroll
              for (int c = 1; c < 4; ++c) tmem_ld32f(lane_addr + scol + 32 * c, v + 32 * c);
              if (look) {
#pragma unroll
                for (int c = 1; c < 4; ++c) tmem_wait32(v + 32 * c);
                look = false;
                if (new_ref(fmaxf(fmaxf(max32(v), max32(v + 32)), fmaxf(max32(v + 64), max32(v + 96)))))
                  continue;   // with the changed logits
              }
              const float r = against(ref);
              uint64_t acc[4] = {0, 0, 0, 0};
              exp32<false>(v, a.sl2, r, pk, acc);
#pragma unroll
              for (int c = 1; c < 4; ++c) tmem_wait32(v + 32 * c);
#pragma unroll
              for (int c = 1; c < 4; ++c) exp32<false>(v + 32 * c, a.sl2, r, pk + 16 * c, acc);
              sum = total(acc);
              look = __any_sync(0xffffffffu, live && sum + l >= kMaxSum);
              if (again || !look) break;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_st16(lane_addr + scol + 32 * c, pk + 16 * c);
          }
          if (k > 0 && __any_sync(0xffffffffu, f != 1.f)) {
            ok = done(n - NQ, false);
            if (!ok) break;
            scale_row(lane_addr + ocol, f);
          }
          l = l * f + sum;
          tmem_st_wait();
        }
        tc_fence_before();
        arrive_warp(&bars->p_full[n & 1], lane);
        if (edge) {   // after the arrival: the product with V waits for the search as well
          ok = wait_warp(&bars->searched[edges & 3], (edges >> 2) & 1, abort_flag);
          if (!ok) break;
          const uint4 b = bad[min(e, kMaxEdges - 1)];
          any_bad |= (b.x | b.y | b.z | b.w) != 0;
          ++e;
          ++edges;
        }
      }
      if (!ok) break;
      // ------------------------------------------------------------ the rows' results
      ok = done(n - NQ, true);
      if (!ok) break;
      tc_fence_after();
      if (!warp_live) continue;
      if (__any_sync(0xffffffffu, any_bad)) {
        const Item item = it;   // copies: what a call takes by reference is in memory for good
        const RowVis seen = vis;
        add_bad(a, item, sg.off, sg.cnt, seen, bad, live, lane_addr + ocol);
      }
      if (sg.whole()) {
        const float f = l == 0.f ? 0.f : 1.f / l;
        const int dst = (it.u * a.g + h) * a.t + i;   // fits 32 bits
        int rows[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          rows[j] = __shfl_sync(0xffffffffu, live ? dst : -1, 8 * j + (lane >> 2));
        uint8_t* stage = sm + Lay::kOffStage + (warp - 4) * 2048;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float o[32];
          tmem_ld32f(lane_addr + ocol + 32 * c, o);
          tmem_wait32(o);
          uint4 x[4];
#pragma unroll
          for (int y = 0; y < 4; ++y)
            x[y] = make_uint4(pack_bf16(o[8 * y] * f, o[8 * y + 1] * f),
                              pack_bf16(o[8 * y + 2] * f, o[8 * y + 3] * f),
                              pack_bf16(o[8 * y + 4] * f, o[8 * y + 5] * f),
                              pack_bf16(o[8 * y + 6] * f, o[8 * y + 7] * f));
          store_rows(stage, lane, x, rows, (uint8_t*)a.out + 64 * c, kD * 2);
        }
        if (live && a.lse) a.lse[dst] = row_lse(ref, l);
      } else {
        const int slot = sg.slot(blockIdx.x), r = w * a.T * a.g + row;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float o[32];
          tmem_ld32f(lane_addr + ocol + 32 * c, o);
          tmem_wait32(o);
          float4* p = part4(a, slot, 8 * c, r);
#pragma unroll
          for (int y = 0; y < 8; ++y)
            if (live) p[(size_t)y * a.rows] = make_float4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
          __syncwarp();   // the next TMEM load is the whole warp's
        }
        if (live) a.pml[(size_t)slot * a.rows + r] = make_float2(ref, l);
      }
      tc_fence_before();
    }
    if (!ok) err = GRKV_ERR_TIMEOUT;
  }
  if (err) plan->err = err;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
  if (tid == 0) {
    AttendRec rec = plan->rec;
    rec.err = bars->abort ? GRKV_ERR_TIMEOUT : plan->err;
    a.rec[blockIdx.x] = rec;
  }
}

template <int NQ, typename A>
cudaError_t launch_tc(const A& a, const CUtensorMap& mq, const CUtensorMap& mk,
                      const CUtensorMap& mv, int G, cudaStream_t st) {
  auto kern = k_attend_tc<NQ, A>;
  const uint32_t smem = TcLayout<NQ>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_kernel(false, 1, kern, dim3(G), TcLayout<NQ>::kThreads, smem, st, mq, mk, mv, a);
}

}  // namespace

cudaError_t launch_attend_tc(const CacheShape& s, const AttendArgs& a, bool cross, int G, cudaStream_t st) {
  CUtensorMap mq, mk, mv;
  if (!encode_bf16_3d(&mq, a.q, kD, s.t, (uint64_t)s.U * s.g, 64, a.T, s.g) ||
      !encode_bf16_3d(&mk, a.k, kD, s.page, s.P, 64, s.page) ||
      !encode_bf16_3d(&mv, a.v, kD, s.page, s.P, 64, s.page))
    return cudaErrorInvalidValue;
  auto launch = [&](const auto& x) {
    return a.nq == 1 ? launch_tc<1>(x, mq, mk, mv, G, st) : launch_tc<2>(x, mq, mk, mv, G, st);
  };
  return cross ? launch(CrossArgs{a}) : launch(a);
}

}  // namespace grkv
