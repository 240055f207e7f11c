// Device code of the rotary positions: the angles of a lane's elements and the rotation of a row.
//
// A row's first rotary_dim elements are pairs of coordinates, (i, i + rotary_dim / 2) in the halves layout, (2 i, 2 i + 1) in
// the pairs layout; pair i of a token at position p is turned by p * f_i radians (f_i: rope_frequencies, fs_rope.hip).
//
// Only the angle's fraction of a turn matters, and it is found exactly: f_i / 2 pi is kept as a 64-bit fraction, p times it
// modulo one turn is an integer product modulo 2^64.  Its error is below p * 2^-65 turns, for every position an int32 can hold
// less than fp32's rounding of the sine; the same product in fp32 is off by 0.06 radians at position 10^6.  What is left, an
// eighth of a turn either way, goes through the power series of sine and cosine, whose first omitted terms (x^11 / 11!, x^10 /
// 10! at pi / 4) are 2e-9 and 2.5e-8.
#pragma once

#include "fs_append_rows.h"

namespace fs {
namespace rope {

using append::kEpl;
using append::u32x4;

struct RopeArgs {
  const uint64_t* turns;  // device [rotary_dim / 2]: turns per position, in units of 2^-64
  int32_t dim;            // rotary_dim
  int32_t pairs;          // 1: neighbouring pairs, 0: halves
  float amplitude;
  float direction;        // 1, or -1: the rotation back
};

// cos and sin of frac * 2^-32 turns, each off by at most about 1e-7
__device__ __forceinline__ void cos_sin(uint32_t frac, float& co, float& si) {
  const uint32_t q = (frac + 0x20000000u) >> 30;                     // the nearest quarter of a turn
  const float x = (float)(int32_t)(frac - (q << 30)) * 1.46291807927e-9f;  // 2 pi / 2^32: |x| <= pi / 4
  const float y = x * x;
  float s = __builtin_fmaf(y, 2.7557319224e-6f, -1.9841269841e-4f);  // 1 / 9!, 1 / 7!
  s = __builtin_fmaf(y, s, 8.3333333333e-3f);                        // 1 / 5!
  s = __builtin_fmaf(y, s, -1.6666666667e-1f);                       // 1 / 3!
  s = __builtin_fmaf(x * y, s, x);
  float c = __builtin_fmaf(y, 2.4801587302e-5f, -1.3888888889e-3f);  // 1 / 8!, 1 / 6!
  c = __builtin_fmaf(y, c, 4.1666666667e-2f);                        // 1 / 4!
  c = __builtin_fmaf(y, c, -0.5f);
  c = __builtin_fmaf(y, c, 1.0f);
  const bool odd = q & 1u;
  const float a = odd ? s : c, b = odd ? c : s;
  co = __uint_as_float(__float_as_uint(a) ^ ((q + 1u) << 30 & 0x80000000u));  // quarters 1 and 2
  si = __uint_as_float(__float_as_uint(b) ^ (q << 30 & 0x80000000u));         // quarters 2 and 3
}

// How a row's elements lie over its lanes, eight to a lane.
//   kSplit: the halves layout with rotary_dim a multiple of 8.  Lane l has elements 4 l .. 4 l + 3 and their partners half + 4 l ..,
//     so that it works out four angles for its eight elements and needs nothing from other lanes; lanes behind the rotated
//     part have eight neighbours.
//   kPairs: neighbouring pairs, eight neighbours in every lane.
//   kMixed: the halves layout with any other rotary_dim: eight neighbours in every lane, whose partners are read one by one.
enum Mode { kSplit = 0, kPairs = 1, kMixed = 2 };
inline int mode_of(const RopeArgs& R) { return R.pairs ? kPairs : (R.dim & 7) == 0 ? kSplit : kMixed; }

struct Lane {
  int a, b;   // first of the lane's elements 0 .. 3, of its elements 4 .. 7
  int pair;   // first of its four pairs (kMixed: not used)
  int half;   // pairs of a row
  bool live;  // some of its elements are rotated
};
template <int MODE>
__device__ __forceinline__ Lane lane_of(const RopeArgs& R, int lir) {
  const int half = R.dim >> 1;
  const bool live = lir * kEpl < R.dim;
  if (MODE == kSplit && live) return Lane{4 * lir, half + 4 * lir, 4 * lir, half, true};
  return Lane{kEpl * lir, kEpl * lir + 4, 4 * lir, half, live};
}

// cos and sin of a position's angle, times the amplitude.
__device__ __forceinline__ void angle(const RopeArgs& R, uint64_t turn, int pos, float& co, float& si) {
  const uint32_t frac = __umulhi((uint32_t)pos, (uint32_t)turn) + (uint32_t)pos * (uint32_t)(turn >> 32);
  cos_sin(frac, co, si);
  co *= R.amplitude;
  si *= R.amplitude * R.direction;
}

// The turns of a lane's pairs (kMixed: of its elements), whatever the token.
template <int MODE>
struct Turns {
  static constexpr int n = MODE == kMixed ? 8 : 4;
  uint64_t turn[n];
};
template <int MODE>
__device__ __forceinline__ Turns<MODE> lane_turns(const RopeArgs& R, const Lane& L) {
  Turns<MODE> T;
#pragma unroll
  for (int q = 0; q < Turns<MODE>::n; ++q) {
    const int d = L.a + q, i = MODE != kMixed ? L.pair + q : d < L.half ? d : d - L.half;
    T.turn[q] = i < L.half ? R.turns[i] : 0ull;
  }
  return T;
}

// Cosines and sines of a token's pairs (kMixed: of its elements, the sine with the sign it has there).
template <int MODE>
struct Factors {
  float co[Turns<MODE>::n], si[Turns<MODE>::n];
};
template <int MODE>
__device__ __forceinline__ Factors<MODE> factors(const RopeArgs& R, const Lane& L, const Turns<MODE>& T, int pos) {
  Factors<MODE> F;
#pragma unroll
  for (int q = 0; q < Turns<MODE>::n; ++q) {
    angle(R, T.turn[q], pos, F.co[q], F.si[q]);
    if (MODE == kMixed && L.a + q < L.half) F.si[q] = -F.si[q];
  }
  return F;
}

// The angles of n_tokens tokens and every pair in LDS, worked out by the `threads` of a team: [token][pair] cosines, then sines.
__device__ __forceinline__ int table_row(const RopeArgs& R) { return ((R.dim >> 1) + 3) & ~3; }
template <typename Pos>
__device__ __forceinline__ void fill_table(const RopeArgs& R, float* table, int n_tokens, int thread, int threads, Pos&& pos_of) {
  // a thread keeps to its pair, and as many tokens are worked on side by side as there are threads for
  const int half = R.dim >> 1, row = table_row(R), wide = min(half, threads), side = threads / wide;
  const int t0 = thread / wide;
  if (t0 >= side) return;
  for (int p = thread - t0 * wide; p < half; p += wide) {
    const uint64_t turn = R.turns[p];
#pragma unroll 4
    for (int t = t0; t < n_tokens; t += side) angle(R, turn, pos_of(t), table[t * row + p], table[(n_tokens + t) * row + p]);
  }
}
template <int MODE>
__device__ __forceinline__ Factors<MODE> table_factors(const RopeArgs& R, const Lane& L, const float* table, int n_tokens, int t) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  Factors<MODE> F;
  const int row = table_row(R);
  const float* const co = table + t * row;
  const float* const si = co + n_tokens * row;
  if constexpr (MODE == kMixed) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int d = L.a + q, i = min(d < L.half ? d : d - L.half, L.half - 1);
      F.co[q] = co[i];
      F.si[q] = d < L.half ? -si[i] : si[i];
    }
  } else {  // (a lane's pairs past the last one: not used; its first pair is inside the row)
    const f32x4 c = *reinterpret_cast<const f32x4*>(co + L.pair), s = *reinterpret_cast<const f32x4*>(si + L.pair);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      F.co[q] = c[q];
      F.si[q] = s[q];
    }
  }
  return F;
}

// A lane's eight elements as they are stored, widened where they are used: a row in flight holds half the registers.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <bool kF32>
struct Raw {
  u32x4 w[kF32 ? 2 : 1];
};
// Of the row at element `row` of src.  SPLIT: they are two times four neighbours.
template <bool kF32, bool SPLIT>
__device__ __forceinline__ void load_raw(const void* src, int64_t row, const Lane& L, Raw<kF32>& r) {
  if constexpr (kF32) {
    const float* const p = reinterpret_cast<const float*>(src) + row;
    r.w[0] = *reinterpret_cast<const u32x4*>(p + L.a);
    r.w[1] = *reinterpret_cast<const u32x4*>(p + L.b);
  } else {
    const uint16_t* const p = reinterpret_cast<const uint16_t*>(src) + row;
    if constexpr (SPLIT) {
      const u32x2 a = *reinterpret_cast<const u32x2*>(p + L.a), b = *reinterpret_cast<const u32x2*>(p + L.b);
      r.w[0] = u32x4{a[0], a[1], b[0], b[1]};
    } else {
      r.w[0] = *reinterpret_cast<const u32x4*>(p + L.a);
    }
  }
}
template <bool kF32>
__device__ __forceinline__ void widen(const Raw<kF32>& r, float (&x)[kEpl]) {
#pragma unroll
  for (int q = 0; q < kEpl; ++q) {
    if constexpr (kF32) x[q] = __uint_as_float(r.w[q >> 2][q & 3]);
    else x[q] = append::f16_value((uint16_t)(r.w[0][q >> 1] >> (16 * (q & 1))));
  }
}
// kMixed: the partner of every element of the lane (itself where it is not rotated).
template <bool kF32>
__device__ __forceinline__ void load_partners(const RopeArgs& R, const void* src, int64_t row, const Lane& L, float (&y)[kEpl]) {
#pragma unroll
  for (int q = 0; q < kEpl; ++q) {
    const int d = L.a + q;
    const int64_t at = row + (d < L.half ? d + L.half : d < R.dim ? d - L.half : d);
    if constexpr (kF32) y[q] = reinterpret_cast<const float*>(src)[at];
    else y[q] = append::f16_value(reinterpret_cast<const uint16_t*>(src)[at]);
  }
}

// Turns the lane's elements x of the row at element `row` of src.  An element that is not rotated stays what it is.
template <int MODE, bool kF32>
__device__ __forceinline__ void turn_row(const RopeArgs& R, const Lane& L, const Factors<MODE>& F, float (&x)[kEpl], const void* src, int64_t row) {
  if (!L.live) return;
  if constexpr (MODE == kMixed) {
    float y[kEpl];
    load_partners<kF32>(R, src, row, L, y);
#pragma unroll
    for (int q = 0; q < kEpl; ++q) {
      const float t = __builtin_fmaf(y[q], F.si[q], x[q] * F.co[q]);
      x[q] = L.a + q < R.dim ? t : x[q];
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = MODE == kPairs ? 2 * q : q, k = MODE == kPairs ? 2 * q + 1 : q + 4;
      const float a = x[i], b = x[k];
      const float ya = __builtin_fmaf(-b, F.si[q], a * F.co[q]), yb = __builtin_fmaf(a, F.si[q], b * F.co[q]);
      const bool live = MODE == kSplit || L.pair + q < L.half;
      x[i] = live ? ya : a;
      x[k] = live ? yb : b;
    }
  }
}
// The same for a row by itself, whose factors nobody else needs.  (Its turns are looked up anew at every use: they would be kept in
// registers otherwise.)
template <int MODE, bool kF32>
__device__ __forceinline__ void turn_row_at(const RopeArgs& R, const Lane& L, int pos, float (&x)[kEpl], const void* src, int64_t row) {
  Lane own = L;
  asm volatile("" : "+v"(own.pair), "+v"(own.a));
  turn_row<MODE, kF32>(R, own, factors<MODE>(R, own, lane_turns<MODE>(R, own), pos), x, src, row);
}

// Unit u of groups x parts.  (Wave-uniform: scalar arithmetic, short where the number is.)
__device__ __forceinline__ void split_unit(int64_t u, uint32_t parts, int64_t& group, int& part) {
  if (u <= 0xffffffffll) {
    group = (uint32_t)u / parts;
    part = (int)((uint32_t)u % parts);
  } else {
    group = u / parts;
    part = (int)(u % parts);
  }
}

// The lane's elements stored in the row's type, rounded once; `row`: the row's first element in out.
template <bool kF32, bool SPLIT>
__device__ __forceinline__ void store8(void* out, int64_t row, const Lane& L, const float (&x)[kEpl]) {
  if constexpr (kF32) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    float* const p = reinterpret_cast<float*>(out) + row;
    *reinterpret_cast<f32x4*>(p + L.a) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + L.b) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = (uint32_t)append::f16_bits(x[2 * q]) | ((uint32_t)append::f16_bits(x[2 * q + 1]) << 16);
    uint16_t* const p = reinterpret_cast<uint16_t*>(out) + row;
    if constexpr (SPLIT) {
      *reinterpret_cast<u32x2*>(p + L.a) = u32x2{w[0], w[1]};
      *reinterpret_cast<u32x2*>(p + L.b) = u32x2{w[2], w[3]};
    } else {
      *reinterpret_cast<u32x4*>(p + L.a) = w;
    }
  }
}

}  // namespace rope
}  // namespace fs
