// Device code of appends to FP8_BLOCK models: one power-of-two scale for a block's K (V) rows of a head.
//
// The tokens that a call brings one block of one sequence -- neighbours in the call's list -- are a group; a group and one (KV
// head, K|V) are worked on together: the largest magnitude decides the scale, then the rows are converted.  A scale that grows
// by 2^k takes the codes stored before along: value and new scale are powers of two apart, so that codes keep their bits with
// the exponent k less, and only those that become subnormal are rounded again.
#pragma once

#include "fs_rope_rows.h"

namespace fs {
namespace append {

constexpr int kScaleMin = -15, kScaleMax = 7;  // 2^e: with them every code x scale is an fp16 number

// The least e in range with amax <= 448 * 2^e, 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax);  // (an infinite amax has the largest exponent, a subnormal one the smallest)
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
  return min(max(e, kScaleMin), kScaleMax);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// of a stored scale, whatever its bits are
__device__ __forceinline__ int stored_exponent(float s) {
  return min(max((int)(__float_as_uint(s) >> 23 & 0xFF) - 127, kScaleMin), kScaleMax);
}

// Two E4M3 codes of a word's low (high) half, times `factor`, as codes again: round to nearest even.
__device__ __forceinline__ uint32_t rescale_codes(uint32_t w, float factor) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  const int v = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * factor, a[1] * factor, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * factor, b[1] * factor, v, true);
}

// Eight elements times 2^-e as codes; the sign is the source's own, NaN and overflow become the largest magnitude.
__device__ __forceinline__ u32x2 block_codes(const float (&x)[kEpl], float factor) {
  float y[kEpl];
#pragma unroll
  for (int q = 0; q < kEpl; ++q) y[q] = __builtin_copysignf(fminf(fabsf(x[q] * factor), 448.0f), x[q]);
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], v, true);
  }
  return w;
}

__device__ __forceinline__ float wave_max(float v) {
  v = row_extremum<true>(v, 16);
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return v;
}

// Where token i of the call belongs: its sequence and its block within the sequence; none: seq < 0.
struct TokenKey {
  int seq, block, slot;
};
__device__ __forceinline__ TokenKey token_key(const AppendArgs& A, int64_t i) {
  TokenKey k{-1, 0, 0};
  if (i >= 0 && i < A.n_tokens) {
    const int s = A.seq_idx[i], p = A.pos[i];
    const int b = (int)((uint32_t)p / (uint32_t)A.g.T);
    if (s >= 0 && p >= 0 && b < A.max_blocks) k = TokenKey{s, b, p - b * A.g.T};
  }
  return k;
}

// Rows of a group that a lane keeps between the two passes; a longer group's are read twice.
constexpr int kHeldSteps = 4;

// The groups that begin among tokens chunk .. chunk + A.group_chunk - 1, for one (head, K|V): NWV waves of a workgroup work on a
// group together (all of them call this with the same arguments; s_max: LDS, NWV > 1), or a wave does it alone (NWV = 1).
// R, turns: the rotation of the K rows (ROPE).
template <bool kSrcF32, bool ROPE, int NWV>
__device__ __forceinline__ void append_group_chunk(const AppendArgs& A, const rope::RopeArgs& R, const rope::LaneTurns& turns, int64_t chunk, int kind,
                                                   float* s_max) {
  const int lane = threadIdx.x & 63;
  const int wave = NWV > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const DevGeom& g = A.g;
  const int lpr = 1 << A.lpr_shift, tpw = 64 >> A.lpr_shift, lir = lane & (lpr - 1);
  const int head = kind >> 1, which = kind & 1;
  const void* const src = which ? A.v_new : A.k_new;
  const int64_t stride = which ? A.v_stride : A.k_stride;
  const TokenKey own = token_key(A, lane < A.group_chunk ? chunk + lane : -1), before = token_key(A, chunk + lane - 1);
  uint64_t leaders = __ballot(own.seq >= 0 && !(before.seq == own.seq && before.block == own.block));
  while (leaders) {
    const int first = __builtin_ctzll(leaders);
    leaders &= leaders - 1;
    const int seq = __builtin_amdgcn_readlane(own.seq, first), block = __builtin_amdgcn_readlane(own.block, first);
    const int64_t i0 = chunk + first;
    int64_t n = 0;
    int low = 0x7fffffff, high = -1;  // the group's lowest and highest slot
    for (;;) {
      const TokenKey k = token_key(A, i0 + n + lane);
      const bool in = k.seq == seq && k.block == block;
      const uint64_t m = ~__ballot(in);
      const int more = m ? __builtin_ctzll(m) : 64;
      low = min(low, lane < more ? k.slot : 0x7fffffff);
      high = max(high, lane < more ? k.slot : -1);
      n += more;
      if (more < 64) break;
    }
    low = wave_min(low);
    high = -wave_min(-high);
    const int32_t blk = A.tables[(int64_t)seq * A.max_blocks + block];
    if (blk < 0 || blk >= A.n_blocks) continue;  // (uniform) never write outside the pool
    uint8_t* const chunk_at = A.pool + (uint64_t)blk * g.block_budget + (uint64_t)A.layer * g.layer_bytes + (uint64_t)head * g.head_chunk;
    uint8_t* const rows = chunk_at + (which ? g.kv_tile : 0u);
    float* const scale = reinterpret_cast<float*>(chunk_at + (uint64_t)(g.H - head) * g.head_chunk + 8u * (uint32_t)head) + which;
    const float old_scale = low > 0 ? *scale : 0.f;
    auto load = [&](int64_t t, float (&x)[kEpl]) {  // row of the group's token t, rotated
      const int64_t tok = i0 + t;
      const int64_t row = tok * stride + (int64_t)head * g.D;
      load8<kSrcF32>(src, row + lir * kEpl, x);
      if constexpr (ROPE) {
        if (which == 0 && turns.live) {
          float y[kEpl] = {};
          if (!R.pairs) rope::load_partners<kSrcF32>(src, row, turns, R.dim, y);
          rope::turn_row(R, turns, rope::factors(R, turns, A.pos[tok]), x, y);
        }
      }
    };
    const int64_t t0 = wave * tpw + (lane >> A.lpr_shift);
    constexpr int kTeam = NWV;
    const int step = kTeam * tpw;
    float held[kHeldSteps][kEpl];
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < kHeldSteps; ++s) {
      if (t0 + (int64_t)s * step < n) {
        load(t0 + (int64_t)s * step, held[s]);
#pragma unroll
        for (int q = 0; q < kEpl; ++q) amax = fmaxf(amax, fabsf(held[s][q]));
      }
    }
    for (int64_t t = t0 + (int64_t)kHeldSteps * step; t < n; t += step) {
      float x[kEpl];
      load(t, x);
#pragma unroll
      for (int q = 0; q < kEpl; ++q) amax = fmaxf(amax, fabsf(x[q]));
    }
    amax = wave_max(amax);
    if constexpr (NWV > 1) {
      if (lane == 0) s_max[wave] = amax;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NWV; ++w) amax = fmaxf(amax, s_max[w]);
      __syncthreads();  // (the next group writes s_max again; and every wave has read the old scale)
    }
    const int e_old = low > 0 ? stored_exponent(old_scale) : kScaleMin;
    const int e = max(e_old, scale_exponent(amax));
    if (low > 0 && e > e_old) {  // (uniform) what is stored in front of the new slots and behind them follows the scale
      const float f = power_of_two(e_old - e);
      const int held = g.T - 1 - high + low;
      for (int i = wave * 64 + lane; i < held * lpr; i += NWV * 64) {
        u32x2* const p = reinterpret_cast<u32x2*>(rows) + (i < low * lpr ? i : i + (high + 1 - low) * lpr);
        const u32x2 w = *p;
        *p = u32x2{rescale_codes(w[0], f), rescale_codes(w[1], f)};
      }
    }
    if (wave == 0 && lane == 0) *scale = power_of_two(e);
    const float f = power_of_two(-e);
    auto put = [&](int64_t t, const float (&x)[kEpl]) {
      const int slot = A.pos[i0 + t] - block * g.T;
      kv_store(reinterpret_cast<u32x2*>(rows + (uint64_t)slot * g.row_bytes + lir * kEpl), block_codes(x, f));
    };
#pragma unroll
    for (int s = 0; s < kHeldSteps; ++s)
      if (t0 + (int64_t)s * step < n) put(t0 + (int64_t)s * step, held[s]);
    for (int64_t t = t0 + (int64_t)kHeldSteps * step; t < n; t += step) {
      float x[kEpl];
      load(t, x);
      put(t, x);
    }
  }
}

// All groups of one append, dealt to n_teams teams of NWV waves; this one is number `team`.
template <bool kSrcF32, bool ROPE, int NWV>
__device__ __forceinline__ void append_groups(const AppendArgs& A, const rope::RopeArgs& R, int64_t team, int64_t n_teams, float* s_max) {
  rope::LaneTurns turns{};
  if constexpr (ROPE) turns = rope::lane_turns(R, ((int)threadIdx.x & 63 & ((1 << A.lpr_shift) - 1)) * kEpl);
  const int kinds = 2 * A.g.H;
  const int64_t n_units = (A.n_tokens + A.group_chunk - 1) / A.group_chunk * kinds;
  for (int64_t unit = team; unit < n_units; unit += n_teams)
    append_group_chunk<kSrcF32, ROPE, NWV>(A, R, turns, unit / kinds * A.group_chunk, (int)(unit % kinds), s_max);
}

// BLOCK: the launch has FP8_BLOCK appends (kernels of their own: the groups take twice the registers of the rows).
template <bool kSrcF32, int HP, bool BLOCK>
__device__ __forceinline__ void append_any(const AppendArgs& A, int64_t worker, int64_t n_workers) {
  switch (A.g.dtype) {
    case FS_KV_FP16: append_rows<kSrcF32, FS_KV_FP16, HP>(A, worker, n_workers); break;
    case FS_KV_FP8_E4M3: append_rows<kSrcF32, FS_KV_FP8_E4M3, HP>(A, worker, n_workers); break;
    case FS_KV_INT8: append_rows<kSrcF32, FS_KV_INT8, HP>(A, worker, n_workers); break;
    case FS_KV_FP8_BLOCK:
      if constexpr (BLOCK) append_groups<kSrcF32, false, 1>(A, rope::RopeArgs{}, worker, n_workers, nullptr);
      break;
    default: append_rows<kSrcF32, FS_KV_INT4, HP>(A, worker, n_workers); break;
  }
}

// The workgroup's share of a multi-append launch: `block` = its index among the launch's append workgroups,
// `waves` = waves per workgroup.
template <bool BLOCK>
__device__ __forceinline__ void append_block(const MultiAppendArgs& P, uint32_t block, int waves) {
  int i = 0;
  while (i + 1 < P.n && block >= P.first_block[i + 1]) ++i;
  const AppendArgs& A = P.a[i];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t worker = (int64_t)(block - P.first_block[i]) * waves + wave;
  const int64_t n_workers = (int64_t)(P.first_block[i + 1] - P.first_block[i]) * waves;
  if (A.src_f32) append_any<true, 1, BLOCK>(A, worker, n_workers);
  else append_any<false, 1, BLOCK>(A, worker, n_workers);
}

}  // namespace append
}  // namespace fs
