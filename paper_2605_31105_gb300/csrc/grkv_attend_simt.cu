// Attention over the paged cache on CUDA cores, for fp32 and (GRKV_FORCE_SIMT) bf16: one kernel
// for items of up to 16 rows (decoding), one for row tiles of up to 64, and the join of
// partial results for all kernels.
//
// A row tile of k_attend_simt is up to 64 rows (T tokens x g query heads).  Its keys come in
// sub-tiles of 64 slots, copied page by page to shared memory: K while the last sub-tile's
// values are multiplied, V while the logits are, so that one buffer each does and two CTAs
// fit an SM (one CTA with two buffers each kept the FMA pipe 48% busy with two warps a
// scheduler: 6 units of 1203 slots, 301 queries of 7 heads, 228 us against 220).  A thread of
// 256 holds 4 rows x 4 slots of the logits and then 4 rows x 8 columns of the output; the softmax
// is online: reference (running maximum, log2 units) and sum per row, the output rescaled
// when the reference grows.  Bound by issue (70% of the slots; shared memory reads beside the
// FMAs).  Slots that a row does not see carry p = -1 and are left out of its sums by comparison,
// so whatever lies there (a NaN, an infinity) does not reach the row.
#include <algorithm>

#include "attend_plan.cuh"

namespace grkv {
namespace {

using namespace sm100;

constexpr int kRowTile = 64;   // rows of a tile
constexpr int kSub = 64;       // slots of a sub-tile
constexpr int kThreads = 256;
constexpr int kQStride = kD + 4;        // floats
constexpr int kPStride = kSub / 2 + 4;   // P goes to shared memory in two halves

template <typename T>
struct SimtLayout {
  static constexpr int kStride = kD + 16 / (int)sizeof(T);      // elements of a K or V row
  static constexpr uint32_t kSubBytes = kSub * kStride * sizeof(T);
  static constexpr uint32_t kOffQ = 0;
  static constexpr uint32_t kOffKv = kOffQ + kRowTile * kQStride * 4;   // K, V
  static constexpr uint32_t kOffP = kOffKv + 2 * kSubBytes;
  static constexpr uint32_t kOffAnc = kOffP + kRowTile * kPStride * 4;
  static constexpr uint32_t kOffMask = kOffAnc + kRowTile * (kMaxTree / 8);
  static constexpr uint32_t kOffPlan = kOffMask + kRowTile * 8;
  static constexpr uint32_t kBytes = kOffPlan + ((sizeof(PlanSmem) + 15) & ~15);
};
static_assert(SimtLayout<float>::kBytes <= 113 * 1024, "two CTAs per SM");

__device__ __forceinline__ float4 ld4(const float* p) { return *(const float4*)p; }
__device__ __forceinline__ float4 ld4(const __nv_bfloat16* p) {
  const uint2 v = *(const uint2*)p;
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                     __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) k_attend_simt(AttendArgs a) {
  using Lay = SimtLayout<T>;
  extern __shared__ __align__(16) uint8_t sm[];
  float* qs = (float*)(sm + Lay::kOffQ);
  float* ps = (float*)(sm + Lay::kOffP);
  uint32_t(*anc)[kMaxTree / 32] = (uint32_t(*)[kMaxTree / 32])(sm + Lay::kOffAnc);
  uint32_t(*mask)[2] = (uint32_t(*)[2])(sm + Lay::kOffMask);
  PlanSmem* plan = (PlanSmem*)(sm + Lay::kOffPlan);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const Run run = plan_run(a, plan, kThreads);
  int err = 0;

  for (Segments sg(a, run); sg.more(); sg.next(a)) {
    const Item& it = sg.it;
    const FullTiles full_tiles(a, it, it.tok0, it.ntok);
    T* const kv[2] = {(T*)(sm + Lay::kOffKv), (T*)(sm + Lay::kOffKv + Lay::kSubBytes)};
    // K (0) or V (1) of a sub-tile of the segment: two per slot tile
    auto load = [&](int n, int which) {
      const int x = it.tile(sg.off + (n >> 1)) * kSlotTile + (n & 1) * kSub;
      constexpr int kChunks = kD * (int)sizeof(T) / 16;
      for (int e = tid; e < kSub * kChunks; e += kThreads) {
        const int row = e / kChunks, ch = e % kChunks, slot = x + row, c = slot >> a.shift;
        if (!it.wanted(c << a.shift, (c + 1) << a.shift)) continue;
        const size_t at =
            (((size_t)page_of(a, it.u, c, &err) << a.shift) + (slot & ((1 << a.shift) - 1))) * kD;
        const int off = ch * (16 / (int)sizeof(T));
        cp_async16(smem_u32(kv[which] + row * Lay::kStride + off),
                   (const T*)(which ? a.v : a.k) + at + off);
      }
    };
    const int subs = 2 * sg.cnt;
    load(0, 0);
    // the item's queries; rows that do not exist are zero
    for (int e = tid; e < kRowTile * (kD / 4); e += kThreads) {
      const int r = e / (kD / 4), d = e % (kD / 4) * 4;
      int h, i;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row_of(a, it, 0, r, &h, &i))
        x = ld4((const T*)a.q + (((size_t)it.u * a.g + h) * a.t + i) * kD + d);
      *(float4*)(qs + r * kQStride + d) = x;
    }
    RowVis vis{};
    if (tid < kRowTile) {
      int h, i;
      const bool live = row_of(a, it, 0, tid, &h, &i);
      vis = row_vis(a, it, i, live, sg.end(), anc[tid], &err);
    }
    float m[4], l[4], acc[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[r][c] = 0.f;
    }
    auto ready = [&](int n) {   // before the barrier in front of sub-tile n's logits
      cp_async_wait_all();
      if (tid < kRowTile) {
        const int x = it.tile(sg.off + (n >> 1)) * kSlotTile + (n & 1) * kSub;
        mask[tid][0] = vis.word(x);
        mask[tid][1] = vis.word(x + 32);
      }
    };
    ready(0);
    for (int n = 0; n < subs; ++n) {
      __syncthreads();   // K and the masks are there; the last V has been read
      load(n, 1);
      const bool full = full_tiles.has(it.tile(sg.off + (n >> 1)));
      const T *ks = kv[0], *vs = kv[1];
      float sc[4][4] = {};
      for (int d = 0; d < kD; d += 4) {
        float4 q4[4], k4[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) q4[r] = ld4(qs + (ty * 4 + r) * kQStride + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) k4[j] = ld4(ks + (tx + 16 * j) * Lay::kStride + d);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sc[r][j] = fmaf(q4[r].x, k4[j].x, sc[r][j]);
            sc[r][j] = fmaf(q4[r].y, k4[j].y, sc[r][j]);
            sc[r][j] = fmaf(q4[r].z, k4[j].z, sc[r][j]);
            sc[r][j] = fmaf(q4[r].w, k4[j].w, sc[r][j]);
          }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = ty * 4 + r;
        const uint32_t w0 = mask[row][0], w1 = mask[row][1];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = j < 2 ? w0 : w1;
          const bool see = (w >> ((tx + 16 * j) & 31)) & 1;
          sc[r][j] = see ? sc[r][j] * a.sl2 : -INFINITY;
          top = fmaxf(top, sc[r][j]);
        }
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float M = fmaxf(m[r], top), ref = M == -INFINITY ? 0.f : M;
        const float keep = fast_exp2(m[r] - ref);
        m[r] = M;
        l[r] *= keep;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[r][c] *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = j < 2 ? w0 : w1;
          const bool see = (w >> ((tx + 16 * j) & 31)) & 1;
          const float p = fast_exp2(sc[r][j] - ref);
          if (see) l[r] += p;
          sc[r][j] = see ? p : -1.f;
        }
      }
      cp_async_wait_all();
      __syncthreads();   // V is there, K has been read
      if (n + 1 < subs) load(n + 1, 0);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        __syncwarp();   // a warp writes and reads its own 8 rows
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ps[(ty * 4 + r) * kPStride + tx] = sc[r][2 * half];
          ps[(ty * 4 + r) * kPStride + tx + 16] = sc[r][2 * half + 1];
        }
        __syncwarp();
        const T* vh = vs + half * (kSub / 2) * Lay::kStride;
#pragma unroll 2
        for (int j = 0; j < kSub / 2; j += 4) {
          float4 p4[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) p4[r] = ld4(ps + (ty * 4 + r) * kPStride + j);
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            const float4 va = ld4(vh + (j + jj) * Lay::kStride + tx * 4);
            const float4 vb = ld4(vh + (j + jj) * Lay::kStride + 64 + tx * 4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float p = jj == 0 ? p4[r].x : jj == 1 ? p4[r].y : jj == 2 ? p4[r].z : p4[r].w;
              if (full || !(p < 0.f)) {
                acc[r][0] = fmaf(p, va.x, acc[r][0]);
                acc[r][1] = fmaf(p, va.y, acc[r][1]);
                acc[r][2] = fmaf(p, va.z, acc[r][2]);
                acc[r][3] = fmaf(p, va.w, acc[r][3]);
                acc[r][4] = fmaf(p, vb.x, acc[r][4]);
                acc[r][5] = fmaf(p, vb.y, acc[r][5]);
                acc[r][6] = fmaf(p, vb.z, acc[r][6]);
                acc[r][7] = fmaf(p, vb.w, acc[r][7]);
              }
            }
          }
        }
      }
      if (n + 1 < subs) ready(n + 1);
    }
    const bool whole = sg.whole();
    const int slot = sg.slot(blockIdx.x);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = ty * 4 + r;
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
      int h, i;
      if (!row_of(a, it, 0, row, &h, &i)) continue;
      float4 x0 = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
      float4 x1 = make_float4(acc[r][4], acc[r][5], acc[r][6], acc[r][7]);
      if (whole) {
        const size_t o = ((size_t)it.u * a.g + h) * a.t + i;
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        x0 = make_float4(x0.x * inv, x0.y * inv, x0.z * inv, x0.w * inv);
        x1 = make_float4(x1.x * inv, x1.y * inv, x1.z * inv, x1.w * inv);
        store_row4((T*)a.out + o * kD + tx * 4, x0);
        store_row4((T*)a.out + o * kD + 64 + tx * 4, x1);
        if (a.lse && tx == 0) a.lse[o] = row_lse(m[r], l[r]);
      } else {
        *part4(a, slot, tx, row) = x0;
        *part4(a, slot, 16 + tx, row) = x1;
        if (tx == 0) a.pml[(size_t)slot * a.rows + row] = make_float2(m[r], l[r]);
      }
    }
    __syncthreads();   // the next segment overwrites the queries and both buffers
  }
  if (err) plan->err = err;
  __syncthreads();
  if (tid == 0) {
    AttendRec rec = plan->rec;
    rec.err = plan->err;
    a.rec[blockIdx.x] = rec;
  }
}

// Items of up to R rows, R = 4, 8 or 16: bound by the read of the cache, which goes straight to
// registers.  Each of 8 warps takes 16 slots of a slot tile, 32 / R at a time, a lane
// four dimensions of all of them: R x 32 / R = 32 logits, whose sums over the lanes a
// transpose-reduction of 31 shuffles leaves one to a lane, so that a step has one
// exponential a lane.  The warps' references, sums and outputs are joined at a segment's end.
// Up to 8 rows fit two CTAs on an SM, which keep 16 warps x 8 KB (fp32) in flight: one query of 3
// heads over 32 units of up to 12005 slots, window 4096, takes 31.5 us, 119 MB at 3.8 TB/s, half of
// it starts, the latency of a run's first loads and the join.  (64-row tiles, mostly empty: 134 us.)
constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;

template <int R>
struct FewSmem {
  PlanSmem plan;
  uint32_t anc[kFewWarps][R][kMaxTree / 32];
  float ml[kFewWarps][R][2];
  float4 o[kFewWarps][R][32];
};
static_assert(sizeof(FewSmem<8>) <= 113 * 1024, "two CTAs per SM");

template <typename T, int R>
__global__ void __launch_bounds__(kFewThreads, R <= 8 ? 2 : 1) k_attend_few(AttendArgs a) {
  constexpr int S = 32 / R;   // slots of a step
  extern __shared__ __align__(16) uint8_t sm_few[];
  FewSmem<R>& sm = *(FewSmem<R>*)sm_few;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int my_row = lane / S, my_slot = lane % S;   // of the logit that this lane ends with
  const Run run = plan_run(a, &sm.plan, kFewThreads);
  int err = 0;

  for (Segments sg(a, run); sg.more(); sg.next(a)) {
    const Item& it = sg.it;
    const FullTiles full(a, it, it.tok0, it.ntok);
    float4 q[R], o[R];
    int h, i;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      q[r] = o[r];
      if (row_of(a, it, 0, r, &h, &i))
        q[r] = ld4((const T*)a.q + (((size_t)it.u * a.g + h) * a.t + i) * kD + lane * 4);
    }
    const bool live = row_of(a, it, 0, my_row, &h, &i);
    // one lane of a row works out what the row sees, in the warp's own words
    uint32_t* anc = sm.anc[warp][my_row];
    RowVis vis{0, 0, 0, it.base, nullptr};
    if (my_slot == 0) vis = row_vis(a, it, i, live, sg.end(), anc, &err);
    __syncwarp();
    vis.end_s = __shfl_sync(0xffffffffu, vis.end_s, my_row * S);
    vis.lo = __shfl_sync(0xffffffffu, vis.lo, my_row * S);
    vis.hi = __shfl_sync(0xffffffffu, vis.hi, my_row * S);
    vis.anc = __shfl_sync(0xffffffffu, vis.anc != nullptr, my_row * S) ? anc : nullptr;
    float m = -INFINITY, l = 0.f;   // of row my_row: the same in its S lanes
    const size_t row_off = lane * 4;
    for (int k = 0; k < sg.cnt; ++k) {
      const int tile = it.tile(sg.off + k), x0 = tile * kSlotTile + warp * 16;
      const bool whole = full.has(tile);
      const int c = x0 >> a.shift;
      if (!it.wanted(x0, x0 + 16)) continue;
      const size_t base = (((size_t)page_of(a, it.u, c, &err) << a.shift) + (x0 & ((1 << a.shift) - 1))) * kD;
      const uint32_t seen = whole ? 0xffffffffu : vis.word(x0 & ~31) >> (x0 & 31);
#pragma unroll 1
      for (int s0 = 0; s0 < 16; s0 += S) {
        const bool see = (seen >> (s0 + my_slot)) & 1;
        if (!__any_sync(0xffffffffu, see)) continue;
        float4 kk[S], vv[S];
#pragma unroll
        for (int s = 0; s < S; ++s) kk[s] = ld4((const T*)a.k + base + (size_t)(s0 + s) * kD + row_off);
#pragma unroll
        for (int s = 0; s < S; ++s) vv[s] = ld4((const T*)a.v + base + (size_t)(s0 + s) * kD + row_off);
        float x[32];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int s = 0; s < S; ++s)
            x[r * S + s] = fmaf(q[r].x, kk[s].x, fmaf(q[r].y, kk[s].y, fmaf(q[r].z, kk[s].z, q[r].w * kk[s].w)));
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) {   // lane e ends with the sum of x[e]
          const bool up = (lane & d) != 0;
#pragma unroll
          for (int e = 0; e < d; ++e) {
            const float send = up ? x[e] : x[e + d];
            x[e] = (up ? x[e + d] : x[e]) + __shfl_xor_sync(0xffffffffu, send, d);
          }
        }
        const float logit = see ? x[0] * a.sl2 : -INFINITY;
        float top = logit;
#pragma unroll
        for (int d = S / 2; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float M = fmaxf(m, top), ref = M == -INFINITY ? 0.f : M;
        const float keep = fast_exp2(m - ref), p = see ? fast_exp2(logit - ref) : 0.f;
        m = M;
        l = l * keep + p;
        const bool scale = __any_sync(0xffffffffu, keep != 1.f);
        const uint32_t skip = whole ? 0u : __ballot_sync(0xffffffffu, !see);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (scale) {
            const float f = __shfl_sync(0xffffffffu, keep, r * S);
            o[r].x *= f;
            o[r].y *= f;
            o[r].z *= f;
            o[r].w *= f;
          }
#pragma unroll
          for (int s = 0; s < S; ++s) {
            const float w = __shfl_sync(0xffffffffu, p, r * S + s);
            if ((skip >> (r * S + s)) & 1) continue;   // whatever lies there stays out
            o[r].x = fmaf(w, vv[s].x, o[r].x);
            o[r].y = fmaf(w, vv[s].y, o[r].y);
            o[r].z = fmaf(w, vv[s].z, o[r].z);
            o[r].w = fmaf(w, vv[s].w, o[r].w);
          }
        }
      }
    }
    // a row's sum is spread over its S lanes
#pragma unroll
    for (int d = S / 2; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    if (my_slot == 0) {
      sm.ml[warp][my_row][0] = m;
      sm.ml[warp][my_row][1] = l;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) sm.o[warp][r][lane] = o[r];
    __syncthreads();
    const bool all = sg.whole();
    for (int r = warp; r < R; r += kFewWarps) {
      if (!row_of(a, it, 0, r, &h, &i)) continue;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) M = fmaxf(M, sm.ml[w][r][0]);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        const float f = weight_of(sm.ml[w][r][0], M);
        const float4 y = sm.o[w][r][lane];
        L += f * sm.ml[w][r][1];
        sum.x = fmaf(f, y.x, sum.x);
        sum.y = fmaf(f, y.y, sum.y);
        sum.z = fmaf(f, y.z, sum.z);
        sum.w = fmaf(f, y.w, sum.w);
      }
      if (all) {
        const size_t dst = ((size_t)it.u * a.g + h) * a.t + i;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        store_row4((T*)a.out + dst * kD + lane * 4,
                   make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
        if (a.lse && lane == 0) a.lse[dst] = row_lse(M, L);
      } else {
        const int slot = sg.slot(blockIdx.x);
        *part4(a, slot, lane, r) = sum;
        if (lane == 0) a.pml[(size_t)slot * a.rows + r] = make_float2(M, L);
      }
    }
    __syncthreads();   // the next segment writes the same shared memory
  }
  if (err) sm.plan.err = err;
  __syncthreads();
  if (tid == 0) {
    AttendRec rec = sm.plan.rec;
    rec.err = sm.plan.err;
    a.rec[blockIdx.x] = rec;
  }
}

// The CTA in which the k-th split item starts, or -1 (all lanes of a warp).
__device__ __forceinline__ int split_cta(const AttendArgs& a, int G, int k) {
  constexpr int kTrips = 2 * kMaxAttendSms / 32;
  int u[kTrips];
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int x = 0; x < kTrips; ++x) u[x] = 32 * x + lane < G ? a.rec[32 * x + lane].u : -1;
  int at = -1;
#pragma unroll
  for (int x = 0; x < kTrips; ++x) {
    const uint32_t m = __ballot_sync(0xffffffffu, u[x] >= 0);
    const uint32_t hit = __ballot_sync(0xffffffffu, u[x] >= 0 && __popc(m & ((1u << lane) - 1)) == k);
    if (hit) at = 32 * x + __ffs(hit) - 1;
    k -= __popc(m);
  }
  return at;
}

// Adds up the partial results of the split items, and writes the call's status.  Blocks
// (c, y) take the item that starts in CTA c (kSearch: the c-th split item), a thread four columns
// of a row (an element).  Items of up to 16 rows may have many parts: the one block's threads go over them in groups of
// one thread per element.  Else a thread has one element, or four where there are only two
// parts: eight loads of outputs are in flight.
constexpr int kJoinFewRows = 16;
template <typename T, bool kFewRows, bool kSearch>
__global__ void __launch_bounds__(kFewRows ? 1024 : 256) k_attend_join(AttendArgs a, int G) {
  chain_wait();
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && blockIdx.y == 0 && tid < 32) {
    int err = 0;
    for (int x = tid; x < G; x += 32) err = min(err, a.rec[x].err);
    err = __reduce_min_sync(0xffffffffu, err);
    if (tid == 0) *a.status = err;
  }
  const int c = kSearch ? split_cta(a, G, blockIdx.x) : blockIdx.x;
  if (c < 0) return;
  const AttendRec rec = a.rec[c];
  if (rec.u < 0) return;
  const int elems = a.rows * (kD / 4), parts = rec.last - c + 1;
  const Item it = make_item(a, rec.u, rec.qb);
  // part 0 is in the CTA's second slot, the others in the first of the CTAs after it
  auto slot = [&](int x) { return x == 0 ? 2 * c + 1 : 2 * (c + x); };
  auto store = [&](int row, int c4, float M, float l, float4 o) {
    const int per = a.T * a.g, w = row / per;
    int h, i;
    if (!row_of(a, it, w, row - w * per, &h, &i)) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const size_t dst = ((size_t)it.u * a.g + h) * a.t + i;
    store_row4((T*)a.out + dst * kD + c4 * 4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (a.lse && c4 == 0) a.lse[dst] = row_lse(M, l);
  };
  auto add = [&](float f, float2 ml, float4 p, float* l, float4* o) {
    *l += f * ml.y;
    o->x = fmaf(f, p.x, o->x);
    o->y = fmaf(f, p.y, o->y);
    o->z = fmaf(f, p.z, o->z);
    o->w = fmaf(f, p.w, o->w);
  };
  if (!kFewRows && parts == 2) {
    float2 ml[4][2];
    float4 p[4][2];
    const int e0 = blockIdx.y * 1024 + tid;
    if (blockIdx.y * 1024 >= elems) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int e = min(e0 + 256 * k, elems - 1), c4 = e / a.rows, row = e - c4 * a.rows;
        ml[k][y] = a.pml[(size_t)slot(y) * a.rows + row];
        p[k][y] = *part4(a, slot(y), c4, row);
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = e0 + 256 * k, c4 = e / a.rows;
      const float M = fmaxf(ml[k][0].x, ml[k][1].x);
      float l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int y = 0; y < 2; ++y) add(weight_of(ml[k][y].x, M), ml[k][y], p[k][y], &l, &o);
      if (e < elems) store(e - c4 * a.rows, c4, M, l, o);
    }
    return;
  }
  const int groups = kFewRows ? 1024 / elems : 1;
  const int e = kFewRows ? tid % elems : blockIdx.y * 256 + tid, grp = kFewRows ? tid / elems : 0;
  if (!kFewRows && e >= elems) return;
  const int c4 = e / a.rows, row = e - c4 * a.rows;
  constexpr int kUnroll = 8;
  float M = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int x = grp; grp < groups && x < parts; x += groups * kUnroll) {   // kUnroll parts to a trip
    float2 ml[kUnroll];
    float4 p[kUnroll];
#pragma unroll
    for (int y = 0; y < kUnroll; ++y) {
      const int z = x + y * groups;
      ml[y] = make_float2(-INFINITY, 0.f);
      p[y] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (z >= parts) continue;
      ml[y] = a.pml[(size_t)slot(z) * a.rows + row];
      p[y] = *part4(a, slot(z), c4, row);
    }
    float top = M;
#pragma unroll
    for (int y = 0; y < kUnroll; ++y) top = fmaxf(top, ml[y].x);
    const float keep = weight_of(M, top);
    M = top;
    l *= keep;
    o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
#pragma unroll
    for (int y = 0; y < kUnroll; ++y) add(weight_of(ml[y].x, M), ml[y], p[y], &l, &o);
  }
  if (kFewRows) {
    __shared__ float4 sum_o[1024];
    __shared__ float2 sum_ml[1024];
    sum_o[tid] = o;
    sum_ml[tid] = make_float2(M, l);
    __syncthreads();
    if (grp > 0) return;
    float top = M;
    for (int x = 1; x < groups; ++x) top = fmaxf(top, sum_ml[x * elems + e].x);
    const float keep = weight_of(M, top);
    M = top;
    l *= keep;
    o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
    for (int x = 1; x < groups; ++x) {
      const float2 ml = sum_ml[x * elems + e];
      add(weight_of(ml.x, M), ml, sum_o[x * elems + e], &l, &o);
    }
  }
  store(row, c4, M, l, o);
}

template <typename T>
cudaError_t launch_join(const AttendArgs& a, int G, cudaStream_t st) {
  count_launches(1);
  if (a.rows <= kJoinFewRows)
    return launch_kernel(true, 1, k_attend_join<T, true, false>, dim3(G), 1024, 0, st, a, G);
  // Blocks look for the CTAs of fewer than 32 items rather than being every CTA's (8 items of 256 rows over
  // 152 CTAs were 4864 blocks, of which 256 had work, and a call took 30.4 us instead of 26.5).
  const int64_t items = (int64_t)a.U * a.QB;
  const unsigned y = (a.rows * (kD / 4) + 255) / 256;
  if (items < 32)
    return launch_kernel(true, 1, k_attend_join<T, false, true>, dim3((unsigned)items, y), 256, 0, st, a, G);
  return launch_kernel(true, 1, k_attend_join<T, false, false>, dim3(G, y), 256, 0, st, a, G);
}

template <typename... Args>
cudaError_t launch_main(void (*kern)(Args...), int G, int threads, uint32_t smem, cudaStream_t st,
                        const Args&... args) {
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_kernel(false, 1, kern, dim3(G), threads, smem, st, args...);
}

template <typename T>
cudaError_t launch_simt(const AttendArgs& a, int G, cudaStream_t st) {
  if (a.rows <= 4) return launch_main(k_attend_few<T, 4>, G, kFewThreads, sizeof(FewSmem<4>), st, a);
  if (a.rows <= 8) return launch_main(k_attend_few<T, 8>, G, kFewThreads, sizeof(FewSmem<8>), st, a);
  if (a.rows <= 16) return launch_main(k_attend_few<T, 16>, G, kFewThreads, sizeof(FewSmem<16>), st, a);
  return launch_main(k_attend_simt<T>, G, kThreads, SimtLayout<T>::kBytes, st, a);
}

}  // namespace

// Tokens and row tiles of an item.  bf16 goes to the tensor cores: tiles of 128 rows, two to
// an item where a unit has more rows than one tile holds.
static void plan_rows(const CacheShape& s, int* T, int* nq) {
  const bool tc = s.dtype == GRKV_BF16 && !s.simt;
  const int most = (tc ? 128 : kRowTile) / s.g;
  *T = std::min(s.t, most);
  *nq = tc && s.t > most ? 2 : 1;
}

// The CUDA-core kernels fit an SM twice, but for k_attend_few with 16 rows.
static int ctas_per_sm(const CacheShape& s, int rows) {
  return (s.dtype == GRKV_F32 || s.simt) && (rows <= 8 || rows > 16) ? 2 : 1;
}

// Two parts a CTA.  Items of 9 to 15 rows have half the CTAs of items of 8, and take what those
// would: a call of fewer tokens never needs more.
size_t attend_part_rows(const CacheShape& s) {
  int T, nq;
  plan_rows(s, &T, &nq);
  const int rows = T * nq * s.g, few = std::min(rows, 8);
  return (size_t)2 * kMaxAttendSms * std::max(rows * ctas_per_sm(s, rows), few * ctas_per_sm(s, few));
}

int64_t attend_tiles(const CacheShape& s) {
  int T, nq;
  plan_rows(s, &T, &nq);
  const int item = nq * T;
  const int64_t cap = (((int64_t)s.cols << s.shift) + kSlotTile - 1) / kSlotTile;
  // with a window: its slots from the first to the last token (in a tree from the base on), the sinks
  const int64_t seen = s.W ? ((int64_t)s.W + s.s + item + kMaxTree) / kSlotTile + 4 : cap;
  return (int64_t)s.U * ((s.t + item - 1) / item) * std::max<int64_t>(1, std::min(cap, seen));
}

cudaError_t launch_attend(const CacheShape& s, const AttendIo& io, char* ws, const CacheWs& L,
                          cudaStream_t st) {
  AttendArgs a{};
  a.q = io.q;
  a.k = io.k;
  a.v = io.v;
  a.table = io.table;
  a.len = io.len;
  a.qlen = io.qlen;
  a.parent = io.parent;
  a.out = io.out;
  a.lse = io.lse;
  a.U = s.U;
  a.g = s.g;
  a.t = s.t;
  a.P = s.P;
  a.shift = s.shift;
  a.cols = s.cols;
  a.W = s.W;
  a.s = s.s;
  a.withhold = s.test_timeout;
  a.sl2 = (float)((double)s.scale * 1.4426950408889634);
  a.rec = (AttendRec*)(ws + L.rec);
  a.pml = (float2*)(ws + L.pml);
  a.po = (float*)(ws + L.po);
  a.status = (int*)(ws + L.status);
  plan_rows(s, &a.T, &a.nq);
  a.QB = (s.t + a.nq * a.T - 1) / (a.nq * a.T);
  a.rows = a.nq * a.T * s.g;
  // two row tiles: an item's start and end take about three tiles' time, 8 K cycles
  a.extra = a.nq == 2 ? 3 : 0;
  a.wide = attend_tiles(s) + (int64_t)s.U * a.QB * a.extra >= 1 << 30;
  const int sms = sm_count();
  if (sms <= 0 || sms > kMaxAttendSms) return cudaErrorInvalidDevice;
  const int G = sms * ctas_per_sm(s, a.rows);
  const bool f32 = s.dtype == GRKV_F32;
  cudaError_t e = f32      ? launch_simt<float>(a, G, st)
                  : s.simt ? launch_simt<__nv_bfloat16>(a, G, st)
                           : launch_attend_tc(s, a, G, st);
  if (e != cudaSuccess) return e;
  return f32 ? launch_join<float>(a, G, st) : launch_join<__nv_bfloat16>(a, G, st);
}

}  // namespace grkv
