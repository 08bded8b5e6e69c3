// Rotary positions on the device: angles, and the pairs of a row that a thread holds.
//
// Pair i of a row at position p is turned by p f_i.  The frequency is kept in turns a position, as
// a 64-bit fraction of one (grkv_rope.turns): p times it, modulo 2^64, is the exact fraction of a
// turn that the angle comes to, for any 32-bit position, with two integer multiplications and no
// range reduction.  (An fp32 product is off by p f 2^-24 radians: 0.008 at position 131072.)
#pragma once

#include <cuda_bf16.h>

#include "grkv_internal.cuh"
#include "sm100.cuh"

namespace grkv {

struct RopeArgs {
  uint64_t turns[kD / 2];   // by pair; 0 behind the rotated ones
  float amp;                // factor of cosine and sine
  int half;                 // pairs that are rotated, rotary / 2
};

// How a thread holds its pairs.  Half, Pairs: a pair of 16-byte vectors, a and b: pairs (a[i], b[i])
// of the half layout, or neighbours in a, then in b, of the interleaved one.  Single: one pair of
// elements, for half layouts whose two halves are not whole vectors (rotary / 2 not a multiple of
// 8 in bf16, 4 in fp32).
enum class Hold { Half, Pairs, Single };

template <typename T, Hold H>
struct Pair {
  static constexpr int kVec = H == Hold::Single ? 1 : 16 / (int)sizeof(T);   // pairs of a thread
  static constexpr int kThreads = kD / 2 / kVec;                            // of a row
};

template <typename T, Hold H>
struct Raw {
  uint4 a, b;
};
template <typename T>
struct Raw<T, Hold::Single> {
  T a, b;
};

// Thread s of a row's kThreads: where its two vectors start, its first pair, and how many of its
// pairs are rotated.  What lies behind the rotated dimensions goes through as it is.
template <typename T, Hold H>
struct Place {
  int a, b, pair, on;
  __device__ __forceinline__ Place(int s, int half) {
    constexpr int V = Pair<T, H>::kVec;
    pair = s * V;
    on = min(max(half - pair, 0), V);
    // (pair - half pairs behind the rotated 2 half elements: element 2 pair)
    const bool split = H != Hold::Pairs && pair < half;
    a = split ? pair : 2 * pair;
    b = split ? half + pair : a + V;
  }
};

// By how many positions a row is turned: `by` forwards, or backwards where sin is negative, which is a's
// factor of the sines; cos, that of the cosines, is a.
struct Turn {
  uint32_t by;
  float cos, sin;
};
__device__ __forceinline__ Turn turn_by(int64_t p, float amp, float sign) {
  return Turn{(uint32_t)(p < 0 ? -p : p), amp, p < 0 ? -amp * sign : amp * sign};
}

// Cosine and sine of the fraction f 2^-32 of a turn.  fp32: the nearest quarter, and a rest of at most an
// eighth of a turn, through the Taylor polynomials of both to the 9th and 10th power (the next terms are below
// 2^-28).  The rest is off by 2^-26.3 turns (2^-28 as an fp32 number, as much again from 2 pi 2^-32, 2^-27.6 from their
// product), cosine and sine by 2^-23.2 (the largest over all 2^32 fractions).  (sincospif over the whole turn, of which
// fp32 holds 2^-25, takes as long: 5.6 us for 5.8 over 25000 rows.)
__device__ __forceinline__ void cos_sin(uint32_t f, float* c, float* s) {
  const uint32_t quarter = (f + (1u << 29)) >> 30;   // 0..3
  const float x = (float)(int32_t)(f - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi 2^-32
  const float z = x * x;
  float a = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  a = fmaf(z, a, 8.33333333e-3f);
  a = fmaf(z, a, -1.66666667e-1f);
  a = fmaf(x * z, a, x);
  float b = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  b = fmaf(z, b, -1.38888889e-3f);
  b = fmaf(z, b, 4.16666667e-2f);
  b = fmaf(z, b, -0.5f);
  b = fmaf(z, b, 1.f);
  const bool odd = quarter & 1;
  *c = __uint_as_float(__float_as_uint(odd ? a : b) ^ (((quarter + 1) & 2) << 30));
  *s = __uint_as_float(__float_as_uint(odd ? b : a) ^ ((quarter & 2) << 30));
}
// bf16: the special function unit's, over one turn around 0.  Its documented errors are 2^-21.4 and 2^-21.2; the angle is
// off by 2^-25 turns as an fp32 number, 2^-26.1 from 2 pi 2^-32 and 2^-25.7 from their product: 2^-20.2 together at
// most (2^-21.1 is the largest over all 2^32 fractions), a 2000th of the output's.  With the polynomials an appended
// chunk takes 9.8 us for 9.1, a streamed one 27.2 for 25.5, 524288 kept rows 88.1 for 87.1.
__device__ __forceinline__ void cos_sin_bf16(uint32_t f, float* c, float* s) {
  __sincosf((float)(int32_t)f * 1.46291807926715968e-9f, s, c);
}

template <typename T, Hold H>
struct Angles {
  static constexpr int kVec = Pair<T, H>::kVec;
  float c[kVec], s[kVec];
  // turns: of the thread's pairs, from RopeArgs or a copy
  __device__ __forceinline__ void set(const uint64_t* turns, const Turn& t) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      // (the lower half rounds the upper one: 2^-33 turns)
      const uint32_t f = (uint32_t)((turns[i] * t.by + 0x80000000u) >> 32);
      if (sizeof(T) == 4) cos_sin(f, &c[i], &s[i]);
      else cos_sin_bf16(f, &c[i], &s[i]);
      c[i] *= t.cos;
      s[i] *= t.sin;
    }
  }
};

template <typename T, Hold H>
__device__ __forceinline__ Raw<T, H> load_pair(const T* row, const Place<T, H>& at) {
  Raw<T, H> r;
  if constexpr (H == Hold::Single) {
    r.a = row[at.a];
    r.b = row[at.b];
  } else {
    r.a = *(const uint4*)(row + at.a);
    r.b = *(const uint4*)(row + at.b);
  }
  return r;
}
template <typename T, Hold H>
__device__ __forceinline__ void store_pair(T* row, const Place<T, H>& at, const Raw<T, H>& r) {
  if constexpr (H == Hold::Single) {
    row[at.a] = r.a;
    row[at.b] = r.b;
  } else {
    *(uint4*)(row + at.a) = r.a;
    *(uint4*)(row + at.b) = r.b;
  }
}

// The same for rows that are read once and written for later (as a compact's are).
template <typename T, Hold H>
__device__ __forceinline__ Raw<T, H> load_once(const T* row, const Place<T, H>& at) {
  if constexpr (H == Hold::Single) {
    return load_pair<T, H>(row, at);
  } else {
    return Raw<T, H>{__ldcs((const uint4*)(row + at.a)), __ldcs((const uint4*)(row + at.b))};
  }
}
template <typename T, Hold H>
__device__ __forceinline__ void store_once(T* row, const Place<T, H>& at, const Raw<T, H>& r) {
  if constexpr (H == Hold::Single) {
    store_pair<T, H>(row, at, r);
  } else {
    __stcs((uint4*)(row + at.a), r.a);
    __stcs((uint4*)(row + at.b), r.b);
  }
}

__device__ __forceinline__ void rotate2(float& x, float& y, float c, float s) {
  const float u = fmaf(x, c, -(y * s)), v = fmaf(x, s, y * c);
  x = u;
  y = v;
}

// The thread's rotated pairs, products and sums in fp32, rounded once; the others bit for bit.
template <typename T, Hold H>
__device__ __forceinline__ Raw<T, H> rotate(const Raw<T, H>& in, const Place<T, H>& at,
                                            const Angles<T, H>& an) {
  if (at.on == 0) return in;
  Raw<T, H> out = in;
  if constexpr (H == Hold::Single) {
    float x = (float)in.a, y = (float)in.b;
    rotate2(x, y, an.c[0], an.s[0]);
    out.a = (T)x;
    out.b = (T)y;
  } else {
    const uint32_t a[4] = {in.a.x, in.a.y, in.a.z, in.a.w}, b[4] = {in.b.x, in.b.y, in.b.z, in.b.w};
    uint32_t oa[4], ob[4];
    if constexpr (sizeof(T) == 4) {
      if constexpr (H == Hold::Half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = __uint_as_float(a[i]), y = __uint_as_float(b[i]);
          rotate2(x, y, an.c[i], an.s[i]);
          oa[i] = __float_as_uint(x);
          ob[i] = __float_as_uint(y);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t* w = i < 2 ? a + 2 * i : b + 2 * i - 4;
          uint32_t* o = i < 2 ? oa + 2 * i : ob + 2 * i - 4;
          float x = __uint_as_float(w[0]), y = __uint_as_float(w[1]);
          rotate2(x, y, an.c[i], an.s[i]);
          o[0] = i < at.on ? __float_as_uint(x) : w[0];
          o[1] = i < at.on ? __float_as_uint(y) : w[1];
        }
      }
    } else {
      auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
      auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
      if constexpr (H == Hold::Half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x0 = lo(a[i]), x1 = hi(a[i]), y0 = lo(b[i]), y1 = hi(b[i]);
          rotate2(x0, y0, an.c[2 * i], an.s[2 * i]);
          rotate2(x1, y1, an.c[2 * i + 1], an.s[2 * i + 1]);
          oa[i] = sm100::pack_bf16(x0, x1);
          ob[i] = sm100::pack_bf16(y0, y1);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t w = i < 4 ? a[i & 3] : b[i & 3];
          float x = lo(w), y = hi(w);
          rotate2(x, y, an.c[i], an.s[i]);
          const uint32_t o = i < at.on ? sm100::pack_bf16(x, y) : w;
          if (i < 4) oa[i & 3] = o;
          else ob[i & 3] = o;
        }
      }
    }
    out.a = make_uint4(oa[0], oa[1], oa[2], oa[3]);
    out.b = make_uint4(ob[0], ob[1], ob[2], ob[3]);
  }
  return out;
}

}  // namespace grkv
