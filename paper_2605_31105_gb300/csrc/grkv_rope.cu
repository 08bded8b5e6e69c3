// Rotary positions: of rows on their way from a projection to attention, of new keys on their way
// into the pages, of kept keys that change their slots.
//
// All of them move rows (256 bytes of bf16, 512 of fp32) and turn a row's pairs in between: bound
// by memory, for a few tokens by latency.  A thread holds two 16-byte vectors of a row, which
// hold whole pairs, and the cosines and sines of those pairs, which all heads of a token share.
#include <algorithm>
#include <cmath>

#include "cache_rows.cuh"
#include "rope.cuh"

using namespace grkv;

namespace {

// ---------------------------------------------------------------------- the plan
// Radians a position from which a plan is refused.  fp64 leaves 2^-53 of a frequency's turns: less than 2^-45 turns below
// this, nothing of the fraction from 2^53 on; factors far below 1 overflow, too.
constexpr double kMostRadians = 1024;

int make_rope(const grkv_rope_params* p, const double* factors, grkv_rope* rope) {
  if (!p || !rope) return GRKV_ERR_INVALID_ARG;
  if (p->d < 1 || p->rotary < 2 || p->rotary > p->d || p->rotary % 2) return GRKV_ERR_INVALID_ARG;
  if (p->layout != GRKV_ROPE_HALF && p->layout != GRKV_ROPE_PAIRS) return GRKV_ERR_INVALID_ARG;
  if (p->scaling < GRKV_ROPE_PLAIN || p->scaling > GRKV_ROPE_YARN) return GRKV_ERR_INVALID_ARG;
  auto positive = [](double x) { return x > 0 && std::isfinite(x); };
  if (!(p->theta > 1) || !std::isfinite(p->theta)) return GRKV_ERR_INVALID_ARG;
  if (p->scaling != GRKV_ROPE_PLAIN && !positive(p->factor)) return GRKV_ERR_INVALID_ARG;
  if (!(p->amplitude >= 0) || !std::isfinite(p->amplitude)) return GRKV_ERR_INVALID_ARG;
  const bool ramp = p->scaling == GRKV_ROPE_BANDS || p->scaling == GRKV_ROPE_YARN;
  if (ramp && (!positive(p->original) || !(p->low >= 0) || !(p->high >= 0) || !std::isfinite(p->high)))
    return GRKV_ERR_INVALID_ARG;
  if (p->d != kD) return GRKV_ERR_UNSUPPORTED;
  const double pi2 = 6.283185307179586476925, r = p->rotary;
  const double low = p->low != 0 ? p->low : 1;
  const double high = p->high != 0 ? p->high : p->scaling == GRKV_ROPE_YARN ? 32 : 4;
  if (ramp && !(low < high)) return GRKV_ERR_INVALID_ARG;
  double theta = p->theta;
  if (p->scaling == GRKV_ROPE_NTK && p->rotary > 2) theta *= std::pow(p->factor, r / (r - 2));
  auto dim = [&](double turns) {   // the pair that makes `turns` turns over the trained positions
    return r * std::log(p->original / (pi2 * turns)) / (2 * std::log(p->theta));
  };
  double from = 0, to = 1;
  if (p->scaling == GRKV_ROPE_YARN) {
    from = std::max(std::floor(dim(high)), 0.0);
    to = std::min(std::ceil(dim(low)), r - 1);
    to = from + std::max(to - from, 0.001);
  }
  grkv_rope out{};
  out.rotary = p->rotary;
  out.layout = p->layout;
  out.amplitude = (float)(p->amplitude != 0 ? p->amplitude
                          : p->scaling == GRKV_ROPE_YARN && p->factor > 1 ? 0.1 * std::log(p->factor) + 1
                                                                          : 1.0);
  for (int i = 0; i < p->rotary / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / r), keep = 1;
    if (p->scaling == GRKV_ROPE_LINEAR) f /= p->factor;
    if (p->scaling == GRKV_ROPE_BANDS) keep = (p->original * f / pi2 - low) / (high - low);
    if (p->scaling == GRKV_ROPE_YARN) keep = 1 - (i - from) / (to - from);
    if (ramp) {
      keep = std::min(std::max(keep, 0.0), 1.0);
      f *= keep + (1 - keep) / p->factor;
    }
    if (factors) {
      if (!positive(factors[i])) return GRKV_ERR_INVALID_ARG;
      f /= factors[i];
    }
    if (!(f < kMostRadians)) return GRKV_ERR_INVALID_ARG;   // infinities and NaN too
    double t = f / pi2;
    t = std::ldexp(t - std::floor(t), 64);   // at most 2^64 - 2^11: the fraction has 53 bits
    out.turns[i] = (uint64_t)std::round(t);
  }
  if (!(out.amplitude > 0) || std::isinf(out.amplitude)) return GRKV_ERR_INVALID_ARG;
  *rope = out;
  return GRKV_OK;
}

int check_rope(const grkv_rope* r, RopeArgs* a) {
  if (!r || r->rotary < 2 || r->rotary > kD || r->rotary % 2) return GRKV_ERR_INVALID_ARG;
  if (r->layout != GRKV_ROPE_HALF && r->layout != GRKV_ROPE_PAIRS) return GRKV_ERR_INVALID_ARG;
  if (!(r->amplitude > 0) || std::isinf(r->amplitude)) return GRKV_ERR_INVALID_ARG;
  a->half = r->rotary / 2;
  a->amp = r->amplitude;
  for (int i = 0; i < kD / 2; ++i) a->turns[i] = i < a->half ? r->turns[i] : 0;
  return GRKV_OK;
}

// A call f(T, Hold) for the type and layout.
template <typename F>
cudaError_t dispatch(int dtype, const grkv_rope* r, F f) {
  const int vec = dtype == GRKV_F32 ? 4 : 8;
  auto of_type = [&](auto zero) {
    if (r->layout == GRKV_ROPE_PAIRS) return f(zero, std::integral_constant<Hold, Hold::Pairs>{});
    if (r->rotary / 2 % vec == 0) return f(zero, std::integral_constant<Hold, Hold::Half>{});
    return f(zero, std::integral_constant<Hold, Hold::Single>{});
  };
  return dtype == GRKV_F32 ? of_type(0.f) : of_type(__nv_bfloat16());
}

// -------------------------------------------------------------------------- rows
struct RowsArgs {
  const void* in;
  void* out;
  int64_t is[3], os[3];   // strides of sequence, head, token, in elements
  const int32_t *pos, *start;
  int S, H, t;
  float sign;             // -1: transposed
};

// kThreads threads a token and four of its heads, whose rows are on their way while the angles are formed.  Memory:
// 32 heads of 32768 tokens from token by token to head by head, 537 MB, 79.5 us, what a copy takes; with
// all heads of a token to a thread, and its angles formed once, 83.2 (and 8 heads of 16 tokens 2.8 us for 2.2).
constexpr int kRowThreads = 256, kRowHeads = 4;
template <typename T, Hold H>
__global__ void __launch_bounds__(kRowThreads)
    k_rope_rows(const __grid_constant__ RopeArgs r, const __grid_constant__ RowsArgs a) {
  constexpr int kThr = Pair<T, H>::kThreads;
  const int64_t n = (int64_t)blockIdx.x * (kRowThreads / kThr) + threadIdx.x / kThr;
  if (n >= (int64_t)a.S * a.t) return;
  const int s = (int)n / a.t, i = (int)n - s * a.t;   // S t <= 2^30
  const int64_t p = a.pos ? a.pos[n] : (int64_t)(a.start ? a.start[s] : 0) + i;
  const Place<T, H> at(threadIdx.x % kThr, r.half);
  const int h0 = blockIdx.y * kRowHeads, heads = min(a.H - h0, kRowHeads);
  const T* in = (const T*)a.in + s * a.is[0] + h0 * a.is[1] + i * a.is[2];
  T* out = (T*)a.out + s * a.os[0] + h0 * a.os[1] + i * a.os[2];
  Raw<T, H> x[kRowHeads];
#pragma unroll
  for (int j = 0; j < kRowHeads; ++j)
    if (j < heads) x[j] = load_pair<T, H>(in + j * a.is[1], at);
  if (p < 0) return;
  Angles<T, H> an;
  an.set(r.turns + at.pair, turn_by(p, r.amp, a.sign));
#pragma unroll
  for (int j = 0; j < kRowHeads; ++j)
    if (j < heads) store_pair<T, H>(out + j * a.os[1], at, rotate<T, H>(x[j], at, an));
}

// Whether rows of the strides (elements) are whole vectors apart, reach over 2^40 elements at most, and, for outputs,
// are apart at all.
int check_strides(const int64_t* stride, const int64_t* n, int vec, bool apart) {
  for (int x = 0; x < 3; ++x)
    if (n[x] > 1 && stride[x] % vec) return GRKV_ERR_MISALIGNED;
  for (int x = 0; x < 3; ++x)
    if (n[x] > 1 && (stride[x] < 0 || stride[x] > ((int64_t)1 << 40) / (n[x] - 1))) return GRKV_ERR_INVALID_ARG;
  if (!apart) return GRKV_OK;
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
  int64_t end = kD;   // what the dimensions so far reach over
  for (int x : order) {
    if (n[x] <= 1) continue;
    if (stride[x] < end) return GRKV_ERR_INVALID_ARG;
    // an outer dimension must step over all of the inner ones
    end += stride[x] * (n[x] - 1);
  }
  return GRKV_OK;
}

// ------------------------------------------------------------------------ append
struct AppendRopeArgs {
  RowMove m;
  const void *k_new, *v_new, *q;   // q may be null
  void *q_out, *k, *v;
  const int64_t* first;
  long long new_rows;
  const int32_t *table, *pos, *offset;
  int g, parts;
};

// kThreads threads a token's new key and value and up to kPartHeads of its queries' heads, two in flight; more
// heads are parts of their own.  Rows are asked for before the table's entry that says where they go.  Memory:
// 32768 tokens of 4 heads, 100 MB, 19.0 us; a chunk of 16384 8.4 to 9.3 (8.6 where four heads in flight took 10.4, and
// keys and queries in blocks of their own 10.0).
constexpr int kAppendThreads = 128, kAppendHeads = 2, kPartHeads = 4;
template <typename T, Hold H>
__global__ void __launch_bounds__(kAppendThreads)
    k_append_rope(const __grid_constant__ RopeArgs r, const __grid_constant__ AppendRopeArgs a, int* word,
                  int solo) {
  __shared__ CallStatus::Smem shared;
  const CallStatus st(word, &shared, solo);
  constexpr int kThr = Pair<T, H>::kThreads;
  RowMove m = a.m;
  m.status = st.at();
  const int block = blockIdx.x / a.parts, part = blockIdx.x - block * a.parts;
  const int n = block * (kAppendThreads / kThr) + threadIdx.x / kThr;   // U t <= 2^28
  const int u = n / m.t, i = n - u * m.t;
  const int cnt = u < m.tb.U ? rows_of(m, u) : 0;
  if (i < cnt) {
    const Place<T, H> at(threadIdx.x % kThr, r.half);
    // the length as it is: clamped to the table, rows behind it would go over those before
    const long long slot = (long long)m.len[u] - cnt + i;
    const long long f = a.first ? a.first[u] : (long long)u * m.t;
    const bool has = f >= 0 && f <= a.new_rows - 1 - i, keys = part == 0;
    Raw<T, H> k, v, x[kAppendHeads];
    if (has && keys) {
      k = load_pair<T, H>((const T*)a.k_new + (f + i) * kD, at);
      v = load_pair<T, H>((const T*)a.v_new + (f + i) * kD, at);
    }
    const int64_t row = ((int64_t)u * a.g * m.t + i) * kD, step = (int64_t)m.t * kD;
    const int g = a.q ? min(a.g, (part + 1) * kPartHeads) : 0;
    int h = part * kPartHeads;
    auto load = [&]() {
#pragma unroll
      for (int j = 0; j < kAppendHeads; ++j)
        if (h + j < g) x[j] = load_pair<T, H>((const T*)a.q + row + (h + j) * step, at);
    };
    load();
    int64_t p = slot + (a.offset ? a.offset[u] : 0);
    if (a.pos) p = has ? a.pos[f + i] : -1;
    long long to = -1;
    if (keys) {
      if (has && p >= 0 && slot >= 0 && slot < m.tb.cols << m.tb.shift)
        to = pool_row(m.tb, a.table, u, (int)slot, m.status);
      else
        set_status(m.status, GRKV_ERR_INVALID_ARG);
    }
    if (p >= 0) {
      Angles<T, H> an;
      an.set(r.turns + at.pair, turn_by(p, r.amp, 1.f));
      if (to >= 0) {
        store_pair<T, H>((T*)a.k + to * kD, at, rotate<T, H>(k, at, an));
        store_pair<T, H>((T*)a.v + to * kD, at, v);
      }
      while (h < g) {
#pragma unroll
        for (int j = 0; j < kAppendHeads; ++j)
          if (h + j < g)
            store_pair<T, H>((T*)a.q_out + row + (h + j) * step, at, rotate<T, H>(x[j], at, an));
        h += kAppendHeads;
        load();
      }
    }
  }
  st.end();
}

// ----------------------------------------------------------------------- compact
struct CompactRopeArgs {
  RowMove m;
  const int32_t *idx, *table_in, *table_out, *first, *turn;
  void *k, *v;
};

// By how many positions the key of row i of unit u is turned.
__device__ __forceinline__ int64_t turn_of(const CompactRopeArgs& a, int u, int i) {
  const size_t x = (size_t)u * a.m.t + i;
  return a.turn ? a.turn[x] : (int64_t)(a.first ? a.first[u] : 0) + i - a.idx[x];
}

constexpr int kTurnThreads = 128, kTurnRows = 128, kTurnUnroll = 2;

// To other pages.  A block takes up to kTurnRows rows of one unit: a thread a row looks up where it
// comes from and goes to, then kThreads threads a row move them, two rows in flight to a thread.
// (Places looked up by each row's threads, two rows a block's only work: 106 us for 524288 rows.)
template <typename T, Hold H>
__global__ void __launch_bounds__(kTurnThreads)
    k_gather_rope(const __grid_constant__ RopeArgs r, const __grid_constant__ CompactRopeArgs a, int rows,
                  int* word, int solo) {
  constexpr int kThr = Pair<T, H>::kThreads, kStep = kTurnThreads / kThr;
  __shared__ CallStatus::Smem shared;
  __shared__ long long from[kTurnRows], to[kTurnRows];
  __shared__ int by[kTurnRows];
  const CallStatus st(word, &shared, solo);
  RowMove m = a.m;
  m.status = st.at();
  const int per = (m.t + rows - 1) / rows, u = blockIdx.x / per, i0 = (blockIdx.x - u * per) * rows;
  const int len = m.tb.clamped(m.len[u], m.status), n = min(rows, rows_of(m, u) - i0);
  for (int x = threadIdx.x; x < n; x += kTurnThreads) {
    if (!kept_row(m, a.idx, a.table_in, len, a.table_out, a.first, false, u, i0 + x, &from[x], &to[x])) to[x] = -1;
    else by[x] = (int)turn_of(a, u, i0 + x);
  }
  const Place<T, H> at(threadIdx.x % kThr, r.half);
  Angles<T, H> an;
  uint64_t turns[Pair<T, H>::kVec];
#pragma unroll
  for (int x = 0; x < Pair<T, H>::kVec; ++x) turns[x] = r.turns[at.pair + x];
  __syncthreads();
  for (int x0 = threadIdx.x / kThr; x0 < n; x0 += kStep * kTurnUnroll) {
    Raw<T, H> k[kTurnUnroll], v[kTurnUnroll];
    bool has[kTurnUnroll];
#pragma unroll
    for (int j = 0; j < kTurnUnroll; ++j) {
      const int x = x0 + j * kStep;
      has[j] = x < n && to[x] >= 0;
      if (!has[j]) continue;
      k[j] = load_once<T, H>((const T*)a.k + from[x] * kD, at);
      v[j] = load_once<T, H>((const T*)a.v + from[x] * kD, at);
    }
#pragma unroll
    for (int j = 0; j < kTurnUnroll; ++j) {
      const int x = x0 + j * kStep;
      if (!has[j]) continue;
      store_once<T, H>((T*)a.v + to[x] * kD, at, v[j]);
      if (by[x] != 0) {
        an.set(turns, turn_by(by[x], 1.f, 1.f));
        k[j] = rotate<T, H>(k[j], at, an);
      }
      store_once<T, H>((T*)a.k + to[x] * kD, at, k[j]);
    }
  }
  st.end();
}

// In place: a row only moves down, so chunks of rows in ascending order, each read as a whole
// before it is written, never overwrite a row that is still to be read; a chunk's rows lie behind the
// places of the one before, and are read while that is written.  A block owns the same few pairs
// of every row of one unit's keys or values: 128 rows a chunk, or, where SMs hold one block at most, 512.  Bound by
// a chunk's latency: 16384 of 32768 slots of 8 units 74 us (256 rows a chunk 94), 4096 of 8192 of 64 units 70,
// 2048 of 32768 of 256 units 137.
constexpr int kMaxShiftUnits = 1 << 26;   // 16 blocks a unit
template <typename T, Hold H>
struct ShiftPart {
  // threads of a row in a block: 64 bytes of it
  static constexpr int kThr = H == Hold::Single ? 32 / (int)sizeof(T) : 2;
  static constexpr int kParts = Pair<T, H>::kThreads / kThr;
};
template <typename T, Hold H>
__global__ void __launch_bounds__(1024)
    k_shift_rope(const __grid_constant__ RopeArgs r, const __grid_constant__ CompactRopeArgs a, int* word,
                 int solo) {
  constexpr int kThr = ShiftPart<T, H>::kThr, kParts = ShiftPart<T, H>::kParts;
  __shared__ CallStatus::Smem shared;
  const CallStatus st(word, &shared, solo);
  RowMove m = a.m;
  m.status = st.at();
  const int u = blockIdx.x / (2 * kParts), part = blockIdx.x % kParts, rows = blockDim.x / kThr;
  const bool keys = blockIdx.x / kParts % 2 == 0;
  T* pool = (T*)(keys ? a.k : a.v);
  const Place<T, H> at(part * kThr + threadIdx.x % kThr, r.half);
  const int n = rows_of(m, u), len = m.tb.clamped(m.len[u], m.status);
  Angles<T, H> an;
  struct Row {
    Raw<T, H> x;
    T* to;   // null: none
    int by;
  };
  auto load = [&](int base, Row* row) {
    const int i = base + threadIdx.x / kThr;
    long long from, to;
    row->to = nullptr;
    if (i >= n || !kept_row(m, a.idx, a.table_in, len, a.table_in, a.first, true, u, i, &from, &to)) return;
    row->by = keys ? (int)turn_of(a, u, i) : 0;
    if (from == to && row->by == 0) return;
    row->x = load_pair<T, H>(pool + from * kD, at);
    row->to = pool + to * kD;
  };
  auto store = [&](Row* row) {
    if (!row->to) return;
    if (row->by != 0) {
      an.set(r.turns + at.pair, turn_by(row->by, 1.f, 1.f));
      row->x = rotate<T, H>(row->x, at, an);
    }
    store_pair<T, H>(row->to, at, row->x);
  };
  Row even, odd;
  load(0, &even);
  for (int base = 0; base < n; base += 2 * rows) {
    load(base + rows, &odd);
    __syncthreads();   // the even chunk has been read, by all
    store(&even);
    load(base + 2 * rows, &even);
    __syncthreads();
    store(&odd);
  }
  st.end();
}

}  // namespace

extern "C" {

void grkv_rope_params_init(grkv_rope_params* p) {
  if (!p) return;
  *p = grkv_rope_params{kD, kD, GRKV_ROPE_HALF, GRKV_ROPE_PLAIN, 10000.0, 1.0, 0.0, 0.0, 8192.0, 0.0};
}

int grkv_rope_make(const grkv_rope_params* p, const double* factors, grkv_rope* rope) {
  return make_rope(p, factors, rope);
}

int grkv_rope_rows(const grkv_rope* rope, const grkv_rows* s, const void* in, void* out,
                   const int32_t* pos, const int32_t* start, void* stream) {
  RopeArgs r;
  GRKV_TRY(check_rope(rope, &r));
  if (!s || s->seqs < 0 || s->heads < 0 || s->tokens < 0 || s->d < 1) return GRKV_ERR_INVALID_ARG;
  if (s->dtype != GRKV_F32 && s->dtype != GRKV_BF16) return GRKV_ERR_INVALID_ARG;
  if (s->flags & ~GRKV_ROPE_TRANSPOSE) return GRKV_ERR_INVALID_ARG;
  if (pos && start) return GRKV_ERR_INVALID_ARG;
  if (s->d != kD || (int64_t)s->seqs * s->tokens > (int64_t)1 << 30 || s->heads > 1 << 16)
    return GRKV_ERR_UNSUPPORTED;
  const int64_t n[3] = {s->seqs, s->heads, s->tokens};
  if (n[0] == 0 || n[1] == 0 || n[2] == 0) return GRKV_OK;
  GRKV_TRY(check_ptrs({in, out}, 16));
  GRKV_TRY(check_optional(pos, 4));
  GRKV_TRY(check_optional(start, 4));
  const int vec = s->dtype == GRKV_F32 ? 4 : 8;
  GRKV_TRY(check_strides(s->in_stride, n, vec, false));
  GRKV_TRY(check_strides(s->out_stride, n, vec, true));
  if (in == out)
    for (int x = 0; x < 3; ++x)
      if (n[x] > 1 && s->in_stride[x] != s->out_stride[x]) return GRKV_ERR_INVALID_ARG;
  RowsArgs a{};
  a.in = in;
  a.out = out;
  for (int x = 0; x < 3; ++x) {
    a.is[x] = n[x] > 1 ? s->in_stride[x] : 0;
    a.os[x] = n[x] > 1 ? s->out_stride[x] : 0;
  }
  a.pos = pos;
  a.start = start;
  a.S = s->seqs;
  a.H = s->heads;
  a.t = s->tokens;
  a.sign = (s->flags & GRKV_ROPE_TRANSPOSE) ? -1.f : 1.f;
  return cuda_rc(dispatch(s->dtype, rope, [&](auto zero, auto hold) {
    using T = decltype(zero);
    constexpr Hold H = decltype(hold)::value;
    const int per = kRowThreads / Pair<T, H>::kThreads;
    const int64_t blocks = ((int64_t)a.S * a.t + per - 1) / per;
    count_launches(1);
    return launch_kernel(false, 1, k_rope_rows<T, H>,
                         dim3((unsigned)blocks, (unsigned)((a.H + kRowHeads - 1) / kRowHeads)), kRowThreads, 0,
                         (cudaStream_t)stream, r, a);
  }));
}

int grkv_cache_append_rope(const grkv_cache_params* p, const grkv_rope* rope, const void* k_new,
                           const void* v_new, const int64_t* first_row, int64_t new_rows,
                           const int32_t* count, const int32_t* pos, const int32_t* offset,
                           const void* q, void* q_out, const int32_t* table, const int32_t* len,
                           void* k_pages, void* v_pages, void* ws, size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  RopeArgs r;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  GRKV_TRY(check_rope(rope, &r));
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({k_new, v_new, k_pages, v_pages}, 16));
    GRKV_TRY(check_ptrs({table, len}, 4));
  }
  GRKV_TRY(check_optional(first_row, 8));
  if (first_row && new_rows < 0) return GRKV_ERR_INVALID_ARG;
  if (pos && offset) return GRKV_ERR_INVALID_ARG;
  if (!q != !q_out) return GRKV_ERR_INVALID_ARG;
  GRKV_TRY(check_optional(count, 4));
  GRKV_TRY(check_optional(pos, 4));
  GRKV_TRY(check_optional(offset, 4));
  GRKV_TRY(check_optional(q, 16));
  GRKV_TRY(check_optional(q_out, 16));
  cudaStream_t st = (cudaStream_t)stream;
  if (s.U == 0) return clear_status((char*)ws, L, st);
  const RowMove m{table_of(s), s.t, count, len, nullptr};
  const AppendRopeArgs a{m, k_new, v_new, q, q_out, k_pages, v_pages, first_row,
                         first_row ? (long long)new_rows : (long long)s.U * s.t, table, pos, offset, s.g,
                         q ? (s.g + kPartHeads - 1) / kPartHeads : 1};
  return cuda_rc(dispatch(s.dtype, rope, [&](auto zero, auto hold) {
    using T = decltype(zero);
    constexpr Hold H = decltype(hold)::value;
    const int per = kAppendThreads / Pair<T, H>::kThreads;
    const int64_t blocks = ((int64_t)s.U * s.t + per - 1) / per * a.parts;
    const size_t bytes = (size_t)s.U * s.t * (4 + (q ? 2 * s.g : 0)) * kD * sizeof(T);
    return launch_call(k_append_rope<T, H>, blocks, kAppendThreads, bytes, (int*)((char*)ws + L.status), st, r, a);
  }));
}

int grkv_cache_compact_rope(const grkv_cache_params* p, const grkv_rope* rope, const int32_t* idx,
                            const int32_t* keep, const int32_t* first, const int32_t* turn,
                            const int32_t* table_in, const int32_t* len_in, const int32_t* table_out,
                            void* k_pages, void* v_pages, void* ws, size_t ws_bytes, void* stream) {
  CacheShape s;
  CacheWs L;
  RopeArgs r;
  GRKV_TRY(cache_begin(p, ws, ws_bytes, &s, &L));
  GRKV_TRY(check_rope(rope, &r));
  if (s.U > 0) {
    GRKV_TRY(check_ptrs({k_pages, v_pages}, 16));
    GRKV_TRY(check_ptrs({idx, table_in, len_in, table_out}, 4));
  }
  GRKV_TRY(check_optional(keep, 4));
  GRKV_TRY(check_optional(first, 4));
  GRKV_TRY(check_optional(turn, 4));
  cudaStream_t st = (cudaStream_t)stream;
  if (s.U == 0) return clear_status((char*)ws, L, st);
  if (table_in == table_out && s.U > kMaxShiftUnits) return GRKV_ERR_UNSUPPORTED;
  int* word = (int*)((char*)ws + L.status);
  const RowMove m{table_of(s), s.t, keep, len_in, nullptr};
  const CompactRopeArgs a{m, idx, table_in, table_out, first, turn, k_pages, v_pages};
  return cuda_rc(dispatch(s.dtype, rope, [&](auto zero, auto hold) {
    using T = decltype(zero);
    constexpr Hold H = decltype(hold)::value;
    const size_t bytes = (size_t)s.U * s.t * 4 * kD * sizeof(T);
    if (table_in == table_out) {
      const int64_t blocks = (int64_t)s.U * 2 * ShiftPart<T, H>::kParts;
      return launch_call(k_shift_rope<T, H>, blocks, blocks <= sm_count() ? 1024 : 256, bytes, word, st, r, a);
    }
    // rows of a block: fewer where that gives more SMs work
    int rows = kTurnRows;
    auto blocks = [&]() { return (int64_t)s.U * ((s.t + rows - 1) / rows); };
    while (rows > 16 && blocks() < 912) rows /= 2;
    return launch_call(k_gather_rope<T, H>, blocks(), kTurnThreads, bytes, word, st, r, a, rows);
  }));
}

}  // extern "C"
