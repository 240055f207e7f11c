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

// What a lane knows of its eight elements d0 .. d0 + 7, whatever the token: their pairs' turns, and where their partners are.
struct LaneTurns {
  uint64_t turn[kEpl];
  int d0, half;
  bool live;     // some of them are rotated
  bool aligned;  // (uniform) halves: the partners of the eight elements are eight neighbours, 16 bytes aligned
};
__device__ __forceinline__ LaneTurns lane_turns(const RopeArgs& R, int d0) {
  LaneTurns L;
  L.d0 = d0;
  L.half = R.dim >> 1;
  L.live = d0 < R.dim;
  L.aligned = (L.half & 7) == 0;
#pragma unroll
  for (int q = 0; q < kEpl; ++q) {
    const int d = d0 + q;
    const int i = R.pairs ? d >> 1 : d < L.half ? d : d - L.half;
    L.turn[q] = d < R.dim ? R.turns[i] : 0ull;
  }
  return L;
}

// Factors of a token's elements: y = x * co + partner * si.
struct Factors {
  float co[kEpl], si[kEpl];
};
__device__ __forceinline__ Factors factors(const RopeArgs& R, const LaneTurns& L, int pos) {
  Factors F;
  auto one = [&](int q, float& co, float& si) {
    const uint32_t frac = __umulhi((uint32_t)pos, (uint32_t)L.turn[q]) + (uint32_t)pos * (uint32_t)(L.turn[q] >> 32);
    cos_sin(frac, co, si);
    co *= R.amplitude;
    si *= R.amplitude * R.direction;
  };
  if (R.pairs) {  // (uniform) both elements of a pair are this lane's
#pragma unroll
    for (int q = 0; q < kEpl; q += 2) {
      one(q, F.co[q], F.si[q + 1]);
      F.co[q + 1] = F.co[q];
      F.si[q] = -F.si[q + 1];
    }
  } else {
#pragma unroll
    for (int q = 0; q < kEpl; ++q) {
      one(q, F.co[q], F.si[q]);
      if (L.d0 + q < L.half) F.si[q] = -F.si[q];
    }
  }
  return F;
}

// The partners of the lane's elements of the row at element `row` of src (halves layout; pairs are the lane's own).
template <bool kSrcF32>
__device__ __forceinline__ void load_partners(const void* src, int64_t row, const LaneTurns& L, int dim, float (&y)[kEpl]) {
  if (L.aligned) {  // (uniform)
    append::load8<kSrcF32>(src, row + (L.d0 < L.half ? L.d0 + L.half : L.d0 - L.half), y);
  } else {
#pragma unroll
    for (int q = 0; q < kEpl; ++q) {
      const int d = L.d0 + q;
      const int64_t at = row + (d < L.half ? d + L.half : d < dim ? d - L.half : d);
      if (kSrcF32) y[q] = reinterpret_cast<const float*>(src)[at];
      else y[q] = append::f16_value(reinterpret_cast<const uint16_t*>(src)[at]);
    }
  }
}

// x: the lane's elements; y: their partners (halves layout).  An element that is not rotated stays what it is.
__device__ __forceinline__ void turn_row(const RopeArgs& R, const LaneTurns& L, const Factors& F, float (&x)[kEpl], const float (&y)[kEpl]) {
  float z[kEpl];
#pragma unroll
  for (int q = 0; q < kEpl; ++q) z[q] = R.pairs ? x[q ^ 1] : y[q];
#pragma unroll
  for (int q = 0; q < kEpl; ++q) {
    const float t = __builtin_fmaf(z[q], F.si[q], x[q] * F.co[q]);
    x[q] = L.d0 + q < R.dim ? t : x[q];
  }
}

// Eight elements stored in the row's type, rounded once.
template <bool kF32>
__device__ __forceinline__ void store8(void* out, int64_t at, const float (&x)[kEpl]) {
  if (kF32) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4* const p = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at);
    p[0] = f32x4{x[0], x[1], x[2], x[3]};
    p[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = (uint32_t)append::f16_bits(x[2 * q]) | ((uint32_t)append::f16_bits(x[2 * q + 1]) << 16);
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(out) + at) = w;
  }
}

}  // namespace rope
}  // namespace fs
