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
// The reference of a row is its maximum so far, but it is only moved when the tile's maximum is
// more than 8 above it in log2 units: P stays below 2^8 (bf16 keeps its relative
// precision, the fp32 sums have room) and the output, which has to be rescaled in TMEM when
// the reference moves, is hardly ever touched.  P is rounded to bf16 for the product
// with V: a relative 2^-8 a term, of the size of the output's own rounding; the
// sum of a row is taken in fp32 before it.
//
// Slot tiles that every row sees whole take no masks.  In the others the masks of a row are
// four words, and V is searched for non-finite elements first: they are set to zero
// in shared memory (0 x NaN would reach rows that do not see the slot; what was
// never loaded is there too) and added again, at the end, to the rows that do see them.
#include <algorithm>

#include "attend_plan.cuh"
#include "tmap.cuh"

namespace grkv {
namespace {

using namespace sm100;

constexpr int kRows = 128;                                    // rows of a tile, TMEM lanes
constexpr uint32_t kTileBytes = kSlotTile * kD * 2;           // 32 KB
constexpr int kRing = 4;   // tiles in flight: K in the even slots, V in the odd ones
constexpr long long kWaitBudget = 1ll << 32;                  // cycles (~2 s)
constexpr int kMaxEdges = 16;   // masked tiles of a segment: at most 4 at each end of the
                                // window (256 tokens) and one at the sinks' end
constexpr float kSlack = 8.f;   // how far a tile's maximum may exceed the reference (log2)
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

struct TcBars {
  uint64_t ring_full[kRing], ring_empty[kRing];
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2], p_full[2], pv_done[2];
  uint64_t searched[4];   // V of a masked tile has been searched (uses in turn)
  uint64_t drain;
  uint32_t tmem;
  int abort;
};
static_assert(sizeof(TcBars) <= 512, "barrier block");

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

__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, kWaitBudget));
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

__device__ __forceinline__ float max128(const float* v) {
  float m[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    m[c] = max3(v[c], v[4 + c], v[8 + c]);
#pragma unroll
    for (int x = 12; x < 124; x += 8) m[c] = max3(m[c], v[x + c], v[x + 4 + c]);
    m[c] = fmaxf(m[c], v[124 + c]);
  }
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// exp2(v sl2 - ref) of 64 logits as bf16 pairs; the sum (two partial ones) is of the
// values before rounding.  A row that has seen nothing has v = ref = -inf and gets zeros.
__device__ __forceinline__ uint64_t half_exp(const float* v, float sl2, float ref, uint32_t pk[2][16]) {
  const float r = ref == -INFINITY ? 0.f : ref;
  const uint64_t s2 = pack2(sl2, sl2), m2 = pack2(-r, -r);
  uint64_t acc[2] = {0, 0};
#pragma unroll
  for (int x = 0; x < 32; ++x) {
    float p0, p1;
    unpack2(fma2(pack2(v[2 * x], v[2 * x + 1]), s2, m2), p0, p1);
    p0 = fast_exp2(p0);
    p1 = fast_exp2(p1);
    acc[x & 1] = add2(acc[x & 1], pack2(p0, p1));
    pk[x >> 4][x & 15] = pack_bf16(p0, p1);
  }
  return add2(acc[0], acc[1]);
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
__device__ __noinline__ void add_bad(const AttendArgs& a, const Item& it, int off, int cnt,
                                     const RowVis& vis, const uint4* bad, bool live, uint32_t taddr) {
  int err = 0;
  for (int c0 = 0; c0 < kD; c0 += 32) {
    float o[32];
    tmem_ld32f(taddr + c0, o);
    tmem_wait32(o);
    int e = 0;
    for (int k = 0; live && k < cnt; ++k) {
      const int tile = it.tile(off + k);
      if (tile_full(a, it, it.tok0, it.ntok, tile)) continue;
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

template <int NQ>
__global__ void __launch_bounds__(TcLayout<NQ>::kThreads, 1)
    k_attend_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                const __grid_constant__ CUtensorMap tmV, AttendArgs a) {
  using Lay = TcLayout<NQ>;
  extern __shared__ __align__(1024) uint8_t smraw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
  TcBars* bars = (TcBars*)(sm + Lay::kOffBar);
  PlanSmem* plan = (PlanSmem*)(sm + Lay::kOffPlan);
  uint4* bad_all = (uint4*)(sm + Lay::kOffBad);   // [4][kMaxEdges]
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // warp-uniform for the compiler

  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&bars->ring_full[i], 1);
      mbar_init(&bars->ring_empty[i], i & 1 ? 3 : 1);   // V: the product and both searchers
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->q_full[i], 1);
      mbar_init(&bars->q_empty[i], 1);
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->p_full[i], 4);
      mbar_init(&bars->pv_done[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&bars->searched[i], 2);
    mbar_init(&bars->drain, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  plan_run(a, plan, Lay::kThreads);   // ends with a barrier
  tc_fence_after();
  const Run run = plan->run;
  const uint32_t tmem = bars->tmem;
  volatile int* abort_flag = &bars->abort;
  int err = 0;

  if (warp == 0) {
    // -------------------------------------------------------------- producer
    fewer_regs<NQ>();
    if (lane == 0) {
      prefetch_tensormap(&tmQ);
      prefetch_tensormap(&tmK);
      prefetch_tensormap(&tmV);
    }
    const uint64_t keep = l2_evict_normal();
    const int per_tile = kSlotTile >> a.shift;
    const uint32_t page_bytes = 128u << a.shift;   // of one half
    uint32_t issued = 0;
    int seg = 0;
    Ring pos;
    bool ok = true;
    for (Segments sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
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
      for (int k = 0; ok && k < sg.cnt; ++k) {
        const int c = it.tile(sg.off + k) * per_tile + lane;
        const bool mine =
            lane < per_tile && c < a.cols && it.wanted(c << a.shift, (c + 1) << a.shift);
        const int page = mine ? page_of(a, it.u, c, &err) : 0;
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
    fewer_regs<NQ>();
    // Job n is row tile w of a slot tile; it uses S buffer n & 1.
    constexpr uint32_t id_s = idesc_bf16(kRows, kSlotTile, 0, 0);   // S = Q K^T, both K-major
    constexpr uint32_t id_o = idesc_bf16(kRows, kD, 0, 1);          // O += P V, V MN-major
    constexpr uint32_t kTileDesc = kTileBytes >> 4;
    const uint64_t q_desc = sw128_desc(smem_u32(sm + Lay::kOffQ), 16, 1024);
    const uint64_t k_desc = sw128_desc(smem_u32(sm + Lay::kOffRing), 16, 1024);
    const uint64_t v_desc = sw128_desc(smem_u32(sm + Lay::kOffRing), kTileBytes / 2, 1024);
    Segments qs(a, run), vs(a, run);
    Ring kp, vp;
    vp.add(1);
    uint32_t qn = 0, vn = 0;   // jobs whose S / output products have been issued
    int qk = 0, qseg = 0, vk = 0, vseg = 0;
    uint32_t edges = 0;
    bool ok = true;
    auto issue_s = [&]() -> bool {   // the next slot tile's S products: NQ jobs, or one of them
      const int w = NQ == 2 ? (int)(qn & 1) : 0, b = qseg % Lay::kQBufs;
      if (w == 0) {
        if (qk == 0 && !wait_warp(&bars->q_full[b], (qseg / Lay::kQBufs) & 1, abort_flag)) return false;
        if (!wait_warp(&bars->ring_full[kp.slot], kp.phase, abort_flag)) return false;
      }
      tc_fence_after();
      mma8_ss<id_s>(tmem + (qn & 1) * kSlotTile, q_desc + (b * NQ + w) * kTileDesc,
                    k_desc + kp.slot * kTileDesc);
      mma_commit_elect(&bars->s_full[qn & 1]);
      ++qn;
      if (w == NQ - 1) {
        mma_commit_elect(&bars->ring_empty[kp.slot]);
        kp.add(2);
        if (++qk == qs.cnt) {
          mma_commit_elect(&bars->q_empty[b]);
          qk = 0;
          ++qseg;
          qs.next(a);
        }
      }
      return true;
    };
    if (qs.more()) ok = issue_s();
    if (ok && qs.more()) ok = issue_s();
    while (ok && vs.more()) {
      const int w = NQ == 2 ? (int)(vn & 1) : 0;
      ok = wait_warp(&bars->p_full[vn & 1], (vn >> 1) & 1, abort_flag);
      if (ok && w == 0) {
        ok = wait_warp(&bars->ring_full[vp.slot], vp.phase, abort_flag);
        const Item& it = vs.it;
        if (ok && !tile_full(a, it, it.tok0, it.ntok, it.tile(vs.off + vk))) {
          ok = wait_warp(&bars->searched[edges & 3], (edges >> 2) & 1, abort_flag);
          ++edges;
        }
      }
      if (!ok) break;
      tc_fence_after();
      const uint32_t o = tmem + kColO + (NQ == 2 ? w : vseg & 1) * kD, p = tmem + (vn & 1) * kSlotTile;
      const uint64_t v = v_desc + vp.slot * kTileDesc;
      mma8_ts<id_o, false>(o, p, v, vk > 0);
      mma_commit_elect(&bars->pv_done[vn & 1]);
      ++vn;
      if (w == NQ - 1) {
        mma_commit_elect(&bars->ring_empty[vp.slot]);
        vp.add(2);
        if (++vk == vs.cnt) {
          vk = 0;
          ++vseg;
          vs.next(a);
        }
      }
      if (qs.more()) ok = issue_s();   // over the S buffer that the product above reads
    }
    // every MMA issued so far completes before TMEM is released
    mma_commit_elect(&bars->drain);
    volatile int no_abort = 0;
    mbar_wait(&bars->drain, 0, &no_abort, kWaitBudget);
    __syncwarp();
  } else if (warp < 4) {
    // --------------------------------------------------- search of masked tiles' V
    fewer_regs<NQ>();
    // Two warps, two rows a lane.  They pass every V tile in turn, masked or not, and a V slot is
    // not filled again before they have: so a parity always means the use that they are at,
    // and they are ahead of the softmax by at most the ring's two V tiles, which four marks
    // and four segments' words cover.
    uint32_t edges = 0;
    int seg = 0;
    Ring vp;
    vp.add(1);
    bool ok = true;
    for (Segments sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
      const Item& it = sg.it;
      int e = 0;
      for (int k = 0; ok && k < sg.cnt; ++k, vp.add(2)) {
        ok = wait_warp(&bars->ring_full[vp.slot], vp.phase, abort_flag);
        if (!ok) break;
        if (tile_full(a, it, it.tok0, it.ntok, it.tile(sg.off + k))) {
          if (lane == 0) mbar_arrive(&bars->ring_empty[vp.slot]);
          continue;
        }
        uint8_t* tile = sm + Lay::kOffRing + vp.slot * kTileBytes;
        uint32_t* words = (uint32_t*)(bad_all + (seg & 3) * kMaxEdges + e);
#pragma unroll 1
        for (int r = 0; r < 2; ++r) {
          const int q = (warp - 2) * 2 + r;
          const uint32_t bits = __ballot_sync(0xffffffffu, clean_row(tile, q * 32 + lane));
          if (lane == 0 && e < kMaxEdges) words[q] = bits;
          if (bits) fence_proxy_async_smem();
        }
        arrive_warp(&bars->searched[edges & 3], lane);
        if (lane == 0) mbar_arrive(&bars->ring_empty[vp.slot]);
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
    for (Segments sg(a, run); ok && sg.more(); sg.next(a), ++seg) {
      const Item& it = sg.it;
      int h, i;
      const bool live = row_of(a, it, w, row, &h, &i);
      const bool warp_live = __any_sync(0xffffffffu, live);
      const RowVis vis = row_vis(a, it, i, live, anc, &err);
      const int t0 = it.tok0 + w * a.T, nt = min(a.T, it.tok0 + it.ntok - t0);
      uint4* bad = bad_all + (seg & 3) * kMaxEdges;
      float ref = -INFINITY, l = 0.f;
      int e = 0;
      bool any_bad = false;
      const uint32_t ocol = kColO + (NQ == 2 ? w : seg & 1) * kD;
      // the job before this one of the same output, for which its product is waited for
      auto done = [&](uint32_t job) {
        return wait_warp(&bars->pv_done[job & 1], (job >> 1) & 1, abort_flag);
      };
      for (int k = 0; k < sg.cnt; ++k, n += NQ) {
        const int tile = it.tile(sg.off + k);
        const bool edge = !tile_full(a, it, it.tok0, it.ntok, tile);
        const uint32_t scol = (n & 1) * kSlotTile;
        ok = wait_warp(&bars->s_full[n & 1], (n >> 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (warp_live) {
          float v[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32f(lane_addr + scol + 32 * c, v + 32 * c);
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_wait32(v + 32 * c);
          if (!tile_full(a, it, t0, nt, tile)) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t m = vis.word(tile * kSlotTile + 32 * c);
              if (__all_sync(0xffffffffu, m == 0xffffffffu)) continue;
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!((m >> x) & 1)) v[32 * c + x] = -INFINITY;
            }
          }
          const float top = max128(v) * a.sl2;
          if (k == 0) ref = top;
          const bool move = live && top > ref + kSlack;
          if (__any_sync(0xffffffffu, move)) {
            ok = done(n - NQ);
            if (!ok) break;
            tc_fence_after();
            const float f = move ? fast_exp2(ref - top) : 1.f;
            l *= f;
            if (move) ref = top;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              float o[32];
              tmem_ld32f(lane_addr + ocol + 32 * c, o);
              tmem_wait32(o);
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] *= f;
              tmem_st16(lane_addr + ocol + 32 * c, (uint32_t*)o);
              tmem_st16(lane_addr + ocol + 32 * c + 16, (uint32_t*)o + 16);
            }
          }
          uint32_t pk[2][16];
          uint64_t sum = half_exp(v, a.sl2, ref, pk);
          tmem_st16(lane_addr + scol, pk[0]);
          tmem_st16(lane_addr + scol + 32, pk[1]);
          sum = add2(sum, half_exp(v + 64, a.sl2, ref, pk));
          tmem_st16(lane_addr + scol + 64, pk[0]);
          tmem_st16(lane_addr + scol + 96, pk[1]);
          float l0, l1;
          unpack2(sum, l0, l1);
          l += l0 + l1;
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
      ok = done(n - NQ);
      if (!ok) break;
      tc_fence_after();
      if (!warp_live) continue;
      if (__any_sync(0xffffffffu, any_bad))
        add_bad(a, it, sg.off, sg.cnt, vis, bad, live, lane_addr + ocol);
      const bool whole = sg.whole();
      const float f = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      // rows of out and lse, or of the CTA's part; both counts fit 32 bits
      const int dst = whole ? ((it.u * a.g + h) * a.t + i)
                            : sg.slot(blockIdx.x) * a.rows + w * a.T * a.g + row;
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
        if (whole) {
#pragma unroll
          for (int y = 0; y < 4; ++y)
            x[y] = make_uint4(pack_bf16(o[8 * y] * f, o[8 * y + 1] * f),
                              pack_bf16(o[8 * y + 2] * f, o[8 * y + 3] * f),
                              pack_bf16(o[8 * y + 4] * f, o[8 * y + 5] * f),
                              pack_bf16(o[8 * y + 6] * f, o[8 * y + 7] * f));
          store_rows(stage, lane, x, rows, (uint8_t*)a.out + 64 * c, kD * 2);
        } else {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
            for (int y = 0; y < 4; ++y)
              x[y] = *(const uint4*)(o + 16 * hh + 4 * y);
            store_rows(stage, lane, x, rows, (uint8_t*)a.po + 128 * c + 64 * hh, kD * 4);
          }
        }
      }
      if (live) {
        if (!whole)
          a.pml[dst] = make_float2(ref, l);
        else if (a.lse)
          a.lse[dst] = row_lse(ref, l);
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

template <int NQ>
cudaError_t launch_tc(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk,
                      const CUtensorMap& mv, int G, cudaStream_t st) {
  auto kern = k_attend_tc<NQ>;
  const uint32_t smem = TcLayout<NQ>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_kernel(false, 1, kern, dim3(G), TcLayout<NQ>::kThreads, smem, st, mq, mk, mv, a);
}

}  // namespace

cudaError_t launch_attend_tc(const CacheShape& s, const AttendArgs& a, int G, cudaStream_t st) {
  CUtensorMap mq, mk, mv;
  if (!encode_bf16_3d(&mq, a.q, kD, s.t, (uint64_t)s.U * s.g, 64, a.T, s.g) ||
      !encode_bf16_3d(&mk, a.k, kD, s.page, s.P, 64, s.page) ||
      !encode_bf16_3d(&mv, a.v, kD, s.page, s.P, 64, s.page))
    return cudaErrorInvalidValue;
  return a.nq == 1 ? launch_tc<1>(a, mq, mk, mv, G, st) : launch_tc<2>(a, mq, mk, mv, G, st);
}

}  // namespace grkv
