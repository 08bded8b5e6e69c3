// Attention over encoder states in fp32 for 9 rows a unit and more, on the 5th-generation tensor cores: every fp32
// number is three bf16 parts, x = x1 + x2 + x3 (each the nearest to what the ones before leave: 2^-27 of x is
// lost), and a product of two is the six products of parts whose orders add up to four at most (the others are
// 2^-27 of it), summed in fp32 from the smallest on.  Numbers are halved before they are split, so that none
// rounds up to infinity; parts below 2^-126 are lost, so numbers below 2^-100 are less exact.
//
// A row tile is up to 128 rows, a slot tile 64 slots: S = Q K^T in 48 products of K = 16 and 64 columns, 65 cycles
// each, O = P V in 24 of 128 columns, 57 each.  S goes ahead of O by a tile, so that the tensor cores work on one
// while the softmax does the other's (two S and two P buffers).  O is a tile's alone: the sum over tiles is kept in
// registers, where additions round to nearest, against the running maximum (log2 units).
//
// Roles.  Warps 0-3: softmax, a row (a TMEM lane) to a thread, and its output, 128 registers.  Warps 4-11: queries,
// K and V, read from the pages a tile ahead, split, and stored to shared memory as the products want them.  Warp 12
// issues the products.  Of the block's 512 x 128 registers at launch the warpgroups take 128 x (208 + 128 + 128 + 48).
//
// What bounds it: 4.5 K cycles of products a tile, and the code, of which an SM holds little: 7.2 K cycles a tile
// (every role unrolled, and half the loading warps, took 15 K).  The loading warps keep a tile's K and V in 64 of the
// launch's 128 registers, for which the compiler spills 68 bytes stored and 152 loaded (-Xptxas -v).  Runs are planned
// in tiles of 64 slots and an item's start and end as one more (in tiles of 128, 9 rows of one unit of 300 slots took
// 17.8 us for 14.9).  300 queries of 4 heads over 16 units of up to 1203 slots take 55 us (184 on CUDA cores), 77 of 7
// over 6 units 22.4 (47), 24 rows over 64 units of up to 6000 slots 94 (211), 9 over 128 of 1500 58 (96).  Q in TMEM,
// with K and V in two buffers or copied two tiles ahead, was slower (9 rows over 128 units of 8000 slots 243 us, where
// this took 226 then and 217 now), as were parts formed before there is room for them (285).
#include <stddef.h>

#include <algorithm>

#include "attend_plan.cuh"

namespace grkv {
namespace {

using namespace sm100;

constexpr int kSub = SplitArgs::tile;
constexpr int kThreads = 512, kLoaders = 256;   // kLoaders: of queries, K and V
constexpr uint32_t kQPart = 128 * kD * 2;      // 32 KB: two halves of 64 dimensions
constexpr uint32_t kKvPart = kSub * kD * 2;    // 16 KB
constexpr uint32_t kOffQ = 0, kOffK = 3 * kQPart, kOffV = kOffK + 3 * kKvPart, kOffBar = kOffV + 3 * kKvPart,
                   kOffPlan = kOffBar + 256, kSmem = kOffPlan + 1024 + 1024;   // + alignment slack
static_assert(kSmem <= 227 * 1024 && sizeof(PlanSmem) <= 1024, "smem");
constexpr uint32_t kColP = 128, kColO = 384;   // TMEM: S at 0 and 64, P at 128 and 256 (three parts of 32), O
constexpr long long kWaitBudget = 1ll << 32;   // cycles (~2 s)
constexpr long long kTestWaitBudget = 1ll << 22;   // ~2 ms: GRKV_TEST_TIMEOUT's

// Arrivals that complete a phase: 8 loading warps, 4 of the softmax, or 1 where products do.
struct Bars {
  uint64_t k_full, v_full;                                      // 8
  uint64_t o_empty, p_full[2];                                  // 4
  uint64_t k_empty, v_empty, o_full, s_full[2], drain;          // 1
  uint32_t tmem;
  int abort;
};
constexpr int kBars = 11;
static_assert(sizeof(Bars) <= 256 && offsetof(Bars, tmem) == 8 * kBars, "barriers");

// A CTA's slot tiles in order.
struct Cursor {
  Segments<SplitArgs> sg;
  int sub = 0;
  __device__ Cursor(const SplitArgs& a, const Run& run) : sg(a, run) {}
  __device__ bool more() const { return sg.more(); }
  __device__ bool first() const { return sub == 0; }
  __device__ bool last() const { return sub + 1 == sg.cnt; }
  __device__ int slot() const { return (sg.off + sub) * kSub; }
  __device__ void next(const SplitArgs& a) {
    if (++sub < sg.cnt) return;
    sg.next(a);
    sub = 0;
  }
};

__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort, long long budget) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, budget));
}
__device__ __forceinline__ void arrive_warp(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

// Two numbers' three parts, as pairs of bf16.
__device__ __forceinline__ void split2(float x, float y, uint32_t* p) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = pack_bf16(x, y);
    x -= __uint_as_float(p[i] << 16);
    y -= __uint_as_float(p[i] & 0xffff0000u);
  }
}

// Eight numbers of row r, chunk c (of 8 dimensions), halved and split, to a tile whose parts are `part` bytes and
// whose halves of 64 dimensions `half` bytes apart.
__device__ __forceinline__ void store_split(uint8_t* tile, uint32_t part, uint32_t half, int r, int c, const float4& x,
                                            const float4& y) {
  uint32_t w[4][3];
  split2(0.5f * x.x, 0.5f * x.y, w[0]);
  split2(0.5f * x.z, 0.5f * x.w, w[1]);
  split2(0.5f * y.x, 0.5f * y.y, w[2]);
  split2(0.5f * y.z, 0.5f * y.w, w[3]);
  uint8_t* at = tile + (c >> 3) * half + sw128_offset(r, c & 7);
#pragma unroll
  for (int i = 0; i < 3; ++i) *(uint4*)(at + i * part) = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
}

// A lane's part of a K or V tile: chunk c of rows r0 + 16 j.
constexpr int kRowStep = kLoaders / 16, kChunks = kSub / kRowStep;
struct Chunks {
  float4 x[kChunks], y[kChunks];
};
// The pages of a tile's slots, one to a lane (four of 16 slots, or fewer).
__device__ __forceinline__ int pages_of(const SplitArgs& a, const Cursor& cur, int lane, int* err) {
  const int c = (cur.slot() >> a.shift) + lane;
  return lane < max(1, kSub >> a.shift) && c << a.shift < cur.sg.it.L ? page_of(a, cur.sg.it.u, c, err) : 0;
}
__device__ __forceinline__ void load_chunks(const SplitArgs& a, const void* pool, int pages, int x0, int L, int r0,
                                            int c, Chunks* z) {
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    const int r = r0 + kRowStep * j, slot = x0 + r;
    const int page = __shfl_sync(0xffffffffu, pages, (slot >> a.shift) - (x0 >> a.shift));
    const float4* p =
        (const float4*)pool + (((size_t)page << a.shift) + (slot & ((1 << a.shift) - 1))) * (kD / 4) + 2 * c;
    z->x[j] = z->y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (slot < L) {
      z->x[j] = __ldg(p);
      z->y[j] = __ldg(p + 1);
    }
  }
}
__device__ __forceinline__ void store_chunks(uint8_t* tile, int r0, int c, const Chunks& z) {
#pragma unroll
  for (int j = 0; j < kChunks; ++j) store_split(tile, kKvPart, kKvPart / 2, r0 + kRowStep * j, c, z.x[j], z.y[j]);
}

// The K = 16 steps of a product of parts, by one elected lane of a converged warp, whose descriptors advance inside.
// S: both operands K-major, their halves of 64 dimensions 16 and 8 KB apart.
template <uint32_t kIdesc>
__device__ __forceinline__ void mma_s(uint32_t d, uint64_t q, uint64_t k, bool accumulate) {
  asm volatile(
      "{\n .reg .pred e, f, t;\n .reg .b64 a, b;\n"
      " elect.sync _|e, 0xffffffff;\n"
      " setp.ne.b32 f, %4, 0;\n setp.eq.b32 t, 0, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, f;\n"
      " add.u64 a, %1, 2;\n add.u64 b, %2, 2;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 4;\n add.u64 b, %2, 4;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 6;\n add.u64 b, %2, 6;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 1024;\n add.u64 b, %2, 512;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 1026;\n add.u64 b, %2, 514;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 1028;\n add.u64 b, %2, 516;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      " add.u64 a, %1, 1030;\n add.u64 b, %2, 518;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n}\n" ::"r"(d),
      "l"(q), "l"(k), "n"(kIdesc), "r"((uint32_t)accumulate)
      : "memory");
}
// O: P in TMEM, 8 columns a step; V MN-major, 2 KB a step.
template <uint32_t kIdesc>
__device__ __forceinline__ void mma_o(uint32_t d, uint32_t p, uint64_t v, bool accumulate) {
  asm volatile(
      "{\n .reg .pred e, f, t;\n .reg .b64 b;\n .reg .b32 a;\n"
      " elect.sync _|e, 0xffffffff;\n"
      " setp.ne.b32 f, %4, 0;\n setp.eq.b32 t, 0, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, f;\n"
      " add.u32 a, %1, 8;\n add.u64 b, %2, 128;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n"
      " add.u32 a, %1, 16;\n add.u64 b, %2, 256;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n"
      " add.u32 a, %1, 24;\n add.u64 b, %2, 384;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n}\n" ::"r"(d),
      "r"(p), "l"(v), "n"(kIdesc), "r"((uint32_t)accumulate)
      : "memory");
}
// The six products of parts, smallest first: part 4 bits of the left and of the right operand.
constexpr uint32_t kLeft = 0x001102, kRight = 0x010120;
__host__ __device__ constexpr uint32_t part_of(uint32_t parts, int p) { return (parts >> (4 * p)) & 15; }

__global__ void __launch_bounds__(kThreads, 1) k_cross_split(const __grid_constant__ SplitArgs a) {
  extern __shared__ __align__(1024) uint8_t smraw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
  Bars* bars = (Bars*)(sm + kOffBar);
  PlanSmem* plan = (PlanSmem*)(sm + kOffPlan);
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (warp == 0) {
    if (lane < kBars) mbar_init((uint64_t*)bars + lane, lane < 2 ? 8 : lane < 5 ? 4 : 1);
    if (lane == 0) bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 12) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  const Run run = plan_run(a, plan, kThreads);   // ends with a barrier
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  volatile int* abort_flag = &bars->abort;
  // GRKV_TEST_TIMEOUT: CTA 0 never says that its first V has been stored, and soon gives up
  const bool withhold = a.withhold && blockIdx.x == 0;
  const long long budget = withhold ? kTestWaitBudget : kWaitBudget;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return wait_warp(bar, parity & 1, abort_flag, budget); };
  int err = 0;

  if (warp >= 12) {
    // ------------------------------------------------------------- the products
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 12) {
      constexpr uint32_t id_s = idesc_bf16(128, kSub, 0, 0);   // both K-major
      constexpr uint32_t id_o = idesc_bf16(128, kD, 0, 1);     // V MN-major
      const uint64_t q_desc = sw128_desc(smem_u32(sm + kOffQ), 16, 1024);
      const uint64_t k_desc = sw128_desc(smem_u32(sm + kOffK), 16, 1024);
      const uint64_t v_desc = sw128_desc(smem_u32(sm + kOffV), kKvPart / 2, 1024);
      const int tiles = run.left;
      auto issue_s = [&](int n) -> bool {
        if (!wait(&bars->k_full, n)) return false;   // and the queries, if it is a segment's first
        tc_fence_after();
#pragma unroll 1
        for (int p = 0; p < 6; ++p)
          mma_s<id_s>(tmem + (n & 1) * kSub, q_desc + ((part_of(kLeft, p) * kQPart) >> 4),
                      k_desc + ((part_of(kRight, p) * kKvPart) >> 4), p > 0);
        mma_commit_elect(&bars->s_full[n & 1]);
        mma_commit_elect(&bars->k_empty);
        return true;
      };
      bool ok = tiles == 0 || issue_s(0);
      for (int n = 0; ok && n < tiles; ++n) {
        if (n + 1 < tiles) ok = issue_s(n + 1);
        ok = ok && wait(&bars->p_full[n & 1], n >> 1) && wait(&bars->v_full, n) &&
             (n == 0 || wait(&bars->o_empty, n - 1));
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1
        for (int p = 0; p < 6; ++p)
          mma_o<id_o>(tmem + kColO, tmem + kColP + (n & 1) * 128 + part_of(kLeft, p) * 32,
                      v_desc + ((part_of(kRight, p) * kKvPart) >> 4), p > 0);
        mma_commit_elect(&bars->o_full);
        mma_commit_elect(&bars->v_empty);
      }
      // every product issued so far completes before TMEM is released
      mma_commit_elect(&bars->drain);
      volatile int no_abort = 0;
      mbar_wait(&bars->drain, 0, &no_abort, kWaitBudget);
      __syncwarp();
    }
  } else if (warp >= 4) {
    // -------------------------------------------- queries, K (a tile ahead) and V
    const int t = tid - 128, c = t & 15, r0 = t >> 4;
    // K of tile n + 1 is stored once S of tile n has been formed, then V of tile n once O of the one before has;
    // both were asked for a tile earlier, their pages before that.
    Cursor kc(a, run);
    int v_pages = 0, v_slot = 0, v_len = 0;   // of the tile that kc is ahead of
    auto fill_q = [&]() {
      const Item& it = kc.sg.it;
#pragma unroll 2
      for (int j = 0; j < 128 / kRowStep; ++j) {
        const int r = r0 + kRowStep * j;
        int h, i;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (row_of(a, it, 0, r, &h, &i)) {
          const float4* p = (const float4*)a.q + (((size_t)it.u * a.g + h) * a.t + i) * (kD / 4) + 2 * c;
          x = __ldg(p);
          y = __ldg(p + 1);
        }
        store_split(sm + kOffQ, kQPart, kQPart / 2, r, c, x, y);
      }
    };
    Chunks k, v;
    int pages = 0;
    if (kc.more()) {
      pages = pages_of(a, kc, lane, &err);
      load_chunks(a, a.k, pages, kc.slot(), kc.sg.it.L, r0, c, &k);
      load_chunks(a, a.v, pages, kc.slot(), kc.sg.it.L, r0, c, &v);
      fill_q();
      store_chunks(sm + kOffK, r0, c, k);
      fence_proxy_async_smem();
      arrive_warp(&bars->k_full, lane);
      kc.next(a);
      if (kc.more()) {
        pages = pages_of(a, kc, lane, &err);
        load_chunks(a, a.k, pages, kc.slot(), kc.sg.it.L, r0, c, &k);
      }
      for (int n = 0;; ++n) {
        const bool ahead = kc.more();   // tile n + 1
        if (ahead) {
          if (!wait(&bars->k_empty, n)) break;
          if (kc.first()) fill_q();
          store_chunks(sm + kOffK, r0, c, k);
          fence_proxy_async_smem();
          arrive_warp(&bars->k_full, lane);
          v_pages = pages;
          v_slot = kc.slot();
          v_len = kc.sg.it.L;
          kc.next(a);
          if (kc.more()) pages = pages_of(a, kc, lane, &err);
        }
        if (n > 0 && !wait(&bars->v_empty, n - 1)) break;
        store_chunks(sm + kOffV, r0, c, v);
        fence_proxy_async_smem();
        if (!withhold || warp != 4) arrive_warp(&bars->v_full, lane);
        if (!ahead) break;
        load_chunks(a, a.v, v_pages, v_slot, v_len, r0, c, &v);
        if (kc.more()) load_chunks(a, a.k, pages, kc.slot(), kc.sg.it.L, r0, c, &k);
      }
    }
  } else {
    // ------------------------------------------------------- softmax and outputs
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int row = warp * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16);
    const float sl2 = a.sl2;   // halved queries and keys: a logit is four times the product with it (4 sl2 may pass fp32)
    float acc[kD];
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    auto add_output = [&](int n) -> bool {   // tile n's product with V
      if (!wait(&bars->o_full, n)) return false;
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float o[32];
        tmem_ld32f(lane_addr + kColO + 32 * c, o);
        tmem_wait32(o);
#pragma unroll
        for (int x = 0; x < 32; ++x) acc[32 * c + x] += o[x];
      }
      tc_fence_before();
      arrive_warp(&bars->o_empty, lane);
      return true;
    };
    int n = 0;
    for (Cursor cur(a, run); ok && cur.more(); ++n) {
      if (cur.first()) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int x = 0; x < kD; ++x) acc[x] = 0.f;
      }
      const int left = cur.sg.it.L - cur.slot();   // slots of the tile that the unit has
      const uint32_t s_addr = lane_addr + (n & 1) * kSub, p_addr = lane_addr + kColP + (n & 1) * 128;
      ok = wait(&bars->s_full[n & 1], n >> 1);
      if (!ok) break;
      tc_fence_after();
      float top = -INFINITY;
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {   // (not unrolled: the roles' code shares what an SM holds of it)
        float v[32];
        tmem_ld32f(s_addr + 32 * c, v);
        tmem_wait32(v);
#pragma unroll
        for (int x = 0; x < 32; ++x)
          if (32 * c + x < left) top = fmaxf(top, v[x]);
      }
      top = 4.f * __fmul_rn(top, sl2);
      const float to = fmaxf(m, top), f = m == -INFINITY || to == m ? 1.f : fast_exp2(m - to);
      m = to;
      // (an infinite logit makes its row NaN: against infinity, exact products would all weigh nothing)
      const float ref = m == -INFINITY ? 0.f : m == INFINITY ? NAN : m;
      float sum = 0.f;
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        float v[32];
        tmem_ld32f(s_addr + 32 * c, v);
        tmem_wait32(v);
        uint32_t p[3][16];
#pragma unroll
        for (int x = 0; x < 32; ++x) {
          // the product rounded, as the reference's was: an exact one would be off by what rounding took from that
          v[x] = 32 * c + x < left ? fast_exp2(__fmaf_rn(4.f, __fmul_rn(v[x], sl2), -ref)) : 0.f;
          sum += v[x];
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          uint32_t w[3];
          split2(v[2 * x], v[2 * x + 1], w);
          p[0][x] = w[0];
          p[1][x] = w[1];
          p[2][x] = w[2];
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) tmem_st16(p_addr + 32 * i + 16 * c, p[i]);
      }
      l = l * f + sum;
      tmem_st_wait();
      tc_fence_before();
      arrive_warp(&bars->p_full[n & 1], lane);
      // the outputs of the tile before, in the old reference, and, at a segment's end, of this one
      const bool last = cur.last();
      for (int x = cur.first() ? n : n - 1; ok && x <= (last ? n : n - 1); ++x) {
        ok = add_output(x);
        if (x < n && __any_sync(0xffffffffu, f != 1.f)) {
#pragma unroll
          for (int y = 0; y < kD; ++y) acc[y] *= f;
        }
      }
      if (!ok) break;
      if (last) {
        const Item& it = cur.sg.it;
        int h, i;
        if (row_of(a, it, 0, row, &h, &i)) {
          const bool whole = cur.sg.whole();
          const float to = !whole ? 2.f : l == 0.f ? 0.f : 2.f / l;   // the values were halved
          const size_t dst = ((size_t)it.u * a.g + h) * a.t + i, step = whole ? 1 : a.rows;
          const int slot = cur.sg.slot(blockIdx.x);
          float4* p = whole ? (float4*)a.out + dst * (kD / 4) : part4(a, slot, 0, row);
#pragma unroll
          for (int x = 0; x < kD / 4; ++x)
            p[x * step] = make_float4(acc[4 * x] * to, acc[4 * x + 1] * to, acc[4 * x + 2] * to, acc[4 * x + 3] * to);
          if (!whole) a.pml[(size_t)slot * a.rows + row] = make_float2(m, l);
          else if (a.lse) a.lse[dst] = row_lse(m, l);
        }
        __syncwarp();
      }
      cur.next(a);
    }
  }
  if (err) plan->err = err;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 12) tmem_dealloc(tmem, 512);
  if (tid == 0) {
    AttendRec rec = plan->rec;
    rec.err = bars->abort ? GRKV_ERR_TIMEOUT : plan->err;
    a.rec[blockIdx.x] = rec;
  }
}

}  // namespace

// From 9 rows on, where a row tile is filled by a tenth: 9 rows of a unit of 300 slots take 15 us (20 in the CUDA-core
// kernel), of 128 units of 1500 58 (96), of 8000 217 (381); 64 rows 63 (118) and 226 (510).  Up to 8 rows, tiles of the
// CUDA-core kernel that are mostly empty too are faster: 128 units of 1500 slots take 42.
bool cross_is_split(const CacheShape& s) { return s.dtype == GRKV_F32 && !s.simt && s.g * s.t > 8; }

void split_rows(const CacheShape& s, AttendArgs* a) {
  // two tiles of the CUDA-core kernels' 64 rows, whose parts the workspace holds
  a->T = std::min(s.t, 2 * std::min(s.t, 64 / s.g));
  a->T = std::min(a->T, 128 / s.g);
  a->nq = 1;
  a->QB = (s.t + a->T - 1) / a->T;
  a->rows = a->T * s.g;
  a->extra = 1;   // queries and output
  a->wide = 2 * attend_tiles(s) + (int64_t)s.U * a->QB * a->extra >= 1 << 30;   // tiles of half the slots
}

cudaError_t launch_cross_split(const AttendArgs& a, int G, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(k_cross_split, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_kernel(false, 1, k_cross_split, dim3((unsigned)G), kThreads, kSmem, st, SplitArgs{a});
}

}  // namespace grkv
