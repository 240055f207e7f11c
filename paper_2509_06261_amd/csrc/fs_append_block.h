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

// What a call brings one block, and where that is.
struct Group {
  int seq, block;      // (n == 0: no group begins at the token)
  int64_t first, n;    // its tokens in the call's list
  int low, high;       // their lowest and highest slot
  uint8_t* layer;      // the block's layer; null: not a block of the pool
};
// The group that begins at token i0 (it does: see append_groups).
__device__ __forceinline__ Group find_group(const AppendArgs& A, int64_t i0, int seq, int block) {
  const int lane = threadIdx.x & 63;
  Group G{seq, block, i0, 0, 0x7fffffff, -1, nullptr};
  const int32_t blk = A.tables[(int64_t)seq * A.max_blocks + block];
  for (;;) {
    const TokenKey k = token_key(A, i0 + G.n + lane);
    const uint64_t m = ~__ballot(k.seq == seq && k.block == block);
    const int more = m ? __builtin_ctzll(m) : 64;
    G.low = min(G.low, lane < more ? k.slot : 0x7fffffff);
    G.high = max(G.high, lane < more ? k.slot : -1);
    G.n += more;
    if (more < 64) break;
  }
  G.low = wave_min(G.low);
  G.high = -wave_min(-G.high);
  if (blk >= 0 && blk < A.n_blocks)  // never write outside the pool
    G.layer = A.pool + (uint64_t)blk * A.g.block_budget + (uint64_t)A.layer * A.g.layer_bytes;
  return G;
}

// A head's K or V rows in a block, and their scale.
struct BlockRows {
  uint8_t* rows;
  float* scale;
};
__device__ __forceinline__ BlockRows block_rows(const DevGeom& g, uint8_t* layer, int head, int which) {
  return BlockRows{layer + (uint64_t)head * g.head_chunk + (which ? g.kv_tile : 0u),
                   reinterpret_cast<float*>(layer + (uint64_t)g.H * g.head_chunk + 8u * (uint32_t)head) + which};
}

// The codes in front of slots low .. high and behind them times 2^(e_old - e): this thread's share of `threads`.
__device__ __forceinline__ void follow_scale(const AppendArgs& A, uint8_t* rows, int low, int high, int e_old, int e, int thread, int threads) {
  const int lpr = 1 << A.lpr_shift;
  const float f = power_of_two(e_old - e);
  const int held = A.g.T - 1 - high + low;
  for (int i = thread; i < held * lpr; i += threads) {
    u32x2* const p = reinterpret_cast<u32x2*>(rows) + (i < low * lpr ? i : i + (high + 1 - low) * lpr);
    const u32x2 w = *p;
    *p = u32x2{rescale_codes(w[0], f), rescale_codes(w[1], f)};
  }
}

__device__ __forceinline__ float amax8(float m, const float (&x)[kEpl]) {
#pragma unroll
  for (int q = 0; q < kEpl; ++q) m = fmaxf(m, fabsf(x[q]));
  return m;
}
// split: the lane's elements are two times four neighbours.
__device__ __forceinline__ void put_codes(const AppendArgs& A, uint8_t* rows, int slot, const rope::Lane& L, bool split, const float (&x)[kEpl], float f) {
  uint8_t* const row = rows + (uint64_t)(uint32_t)slot * A.g.row_bytes;
  const u32x2 w = block_codes(x, f);
  if (split) {
    kv_store(reinterpret_cast<uint32_t*>(row + L.a), w[0]);
    kv_store(reinterpret_cast<uint32_t*>(row + L.b), w[1]);
  } else {
    kv_store(reinterpret_cast<u32x2*>(row + L.a), w);
  }
}
// The lane's place in the rows of K or V, and their load.  ROPE: how K rows are rotated (rope::Mode), or kPlain.
constexpr int kPlain = -1;
template <int ROPE>
__device__ __forceinline__ rope::Lane block_lane(const rope::RopeArgs& R, int which, int lir) {
  if (ROPE != kPlain && which == 0) return rope::lane_of<ROPE == kPlain ? 0 : ROPE>(R, lir);
  return rope::Lane{kEpl * lir, kEpl * lir + 4, 0, 0, false};
}
template <bool kSrcF32, int ROPE>
__device__ __forceinline__ void load_block_row(const void* src, int64_t row, const rope::Lane& L, int which, rope::Raw<kSrcF32>& x) {
  if (ROPE == rope::kSplit && which == 0) rope::load_raw<kSrcF32, true>(src, row, L, x);
  else rope::load_raw<kSrcF32, false>(src, row, L, x);
}

// A group's rows of `heads` neighbouring heads from h0 on, K or V, by a team of NWV waves (a workgroup; or one wave, NWV = 1): its
// tokens over the team's lanes, lpr lanes to a row, kSteps rows to a lane.  Those stay in registers between the maximum and the
// conversion; the next head's rows are requested before the waves meet for the maximum, or (AHEAD) before this head's are widened, which
// takes registers of their own.  LATE: a group of more rows than that reads the rest twice.  The angles of the tokens that are kept are worked out once for all heads, in LDS.
// s_max: LDS, 2 * NWV floats; table: LDS, table_floats<NWV>() floats.
constexpr int kSteps = 4;
// A lane's eight elements are four pairs; two numbers each.
constexpr int table_floats(int team) { return team * 64 * kSteps * kEpl; }
template <bool kSrcF32, int ROPE, int NWV, bool LATE, bool AHEAD>
__device__ __forceinline__ void append_group(const AppendArgs& A, const rope::RopeArgs& R, const rope::Lane& L, const Group& G, int which, int h0,
                                             int heads, float* s_max, float* table) {
  const int lane = threadIdx.x & 63;
  const int wave = NWV > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const DevGeom& g = A.g;
  const int tpw = 64 >> A.lpr_shift;
  const void* const src = which ? A.v_new : A.k_new;
  const int64_t stride = which ? A.v_stride : A.k_stride;
  const bool turned = ROPE != kPlain && which == 0, split = ROPE == rope::kSplit && which == 0;  // (uniform)
  const int64_t t0 = wave * tpw + (lane >> A.lpr_shift);
  const int step = NWV * tpw;
  int slot[kSteps];
  rope::Raw<kSrcF32> own[kSteps], ahead[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t t = t0 + (int64_t)s * step;
    slot[s] = t < G.n ? A.pos[G.first + t] - G.block * g.T : -1;
  }
  auto request = [&](int head, rope::Raw<kSrcF32> (&to)[kSteps]) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (slot[s] >= 0)
        load_block_row<kSrcF32, ROPE>(src, (G.first + t0 + (int64_t)s * step) * stride + (int64_t)head * g.D, L, which, to[s]);
  };
  request(h0, own);
  int in_table = 0;  // tokens: all that are kept in registers
  if constexpr (ROPE != kPlain) {
    if (turned) {
      in_table = (int)min(G.n, (int64_t)kSteps * step);
      rope::fill_table(R, table, in_table, wave * 64 + lane, NWV * 64, [&](int t) { return A.pos[G.first + t]; });
      if constexpr (NWV > 1) {
        __syncthreads();
      } else {  // (a wave's own LDS operations complete in order; the fence is for the compiler)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    }
  }
  auto late_row = [&](int head, int64_t t, float (&x)[kEpl]) {  // a row that is not kept
    const int64_t row = (G.first + t) * stride + (int64_t)head * g.D;
    rope::Raw<kSrcF32> w;
    load_block_row<kSrcF32, ROPE>(src, row, L, which, w);
    rope::widen<kSrcF32>(w, x);
    if constexpr (ROPE != kPlain) {
      if (turned && L.live) rope::turn_row_at<ROPE, kSrcF32>(R, L, A.pos[G.first + t], x, src, row);
    }
  };
  for (int k = 0; k < heads; ++k) {
    const int head = h0 + k;
    const BlockRows B = block_rows(g, G.layer, head, which);
    const float old_scale = G.low > 0 ? *B.scale : 0.f;
    float amax = 0.f;
    if constexpr (LATE) {
      for (int64_t t = t0 + (int64_t)kSteps * step; t < G.n; t += step) {  // (before the others are wide)
        float y[kEpl];
        late_row(head, t, y);
        amax = amax8(amax, y);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (AHEAD) {
      if (k + 1 < heads) request(head + 1, ahead);
      __builtin_amdgcn_sched_barrier(0);
    }
    float x[kSteps][kEpl];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (slot[s] < 0) continue;
      rope::widen<kSrcF32>(own[s], x[s]);
      if constexpr (ROPE != kPlain) {
        // (read from LDS anew for every head, one row's at a time)
        if (turned && L.live) {
          int t = (int)t0 + s * step;
          asm volatile("" : "+v"(t));
          rope::turn_row<ROPE, kSrcF32>(R, L, rope::table_factors<ROPE>(R, L, table, in_table, t), x[s], src, (G.first + t) * stride + (int64_t)head * g.D);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      amax = amax8(amax, x[s]);
    }
    if (!AHEAD && k + 1 < heads) request(head + 1, own);
    amax = wave_max(amax);
    if constexpr (NWV > 1) {
      float* const m = s_max + (k & 1) * NWV;  // (two of them, in turn: a wave is at most one barrier ahead)
      if (lane == 0) m[wave] = amax;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NWV; ++w) amax = fmaxf(amax, m[w]);
    }
    const int e_old = G.low > 0 ? stored_exponent(old_scale) : kScaleMin;
    const int e = max(e_old, scale_exponent(amax));
    if (G.low > 0 && e > e_old) follow_scale(A, B.rows, G.low, G.high, e_old, e, wave * 64 + lane, NWV * 64);  // (uniform)
    if (wave == 0 && lane == 0) *B.scale = power_of_two(e);
    const float f = power_of_two(-e);
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (slot[s] >= 0) put_codes(A, B.rows, slot[s], L, split, x[s], f);
    if constexpr (LATE) {
      for (int64_t t = t0 + (int64_t)kSteps * step; t < G.n; t += step) {
        float y[kEpl];
        late_row(head, t, y);
        put_codes(A, B.rows, A.pos[G.first + t] - G.block * g.T, L, split, y, f);
      }
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) own[s] = ahead[s];
    }
  }
  if constexpr (NWV > 1) __syncthreads();  // (the next group's maxima and table)
}

// Place of the k-th (from 0) set bit of m, which has more than k.
__device__ __forceinline__ int nth_bit(uint64_t m, int k) {
  int at = 0;
#pragma unroll
  for (int w = 32; w; w >>= 1) {
    const int c = __popcll(m >> at & ((1ull << w) - 1));
    if (c <= k) {
      k -= c;
      at += w;
    }
  }
  return at;
}

// The groups of one token each among those of a chunk (bits of `singles`): a token's row of one head per lpr lanes, all at once.
template <bool kSrcF32, int ROPE, int NWV>
__device__ __forceinline__ void append_singles(const AppendArgs& A, const rope::RopeArgs& R, const rope::Lane& L, int64_t chunk, uint64_t singles, int which,
                                               int h0, int heads) {
  const int lane = threadIdx.x & 63;
  const int wave = NWV > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const DevGeom& g = A.g;
  const int lpr = 1 << A.lpr_shift, lir = lane & (lpr - 1), rpw = 64 >> A.lpr_shift;
  const void* const src = which ? A.v_new : A.k_new;
  const bool split = ROPE == rope::kSplit && which == 0;
  const int n = __popcll(singles) * heads;
  for (int base = 0; base < n; base += NWV * rpw) {  // (uniform)
    const int item = base + wave * rpw + (lane >> A.lpr_shift);
    const bool in = item < n;
    const int which_one = in ? item / heads : 0, head = h0 + (in ? item - which_one * heads : 0);
    const int64_t tok = chunk + nth_bit(singles, which_one);
    const int64_t row = tok * (which ? A.v_stride : A.k_stride) + (int64_t)head * g.D;
    rope::Raw<kSrcF32> w;
    if (in) load_block_row<kSrcF32, ROPE>(src, row, L, which, w);
    const TokenKey k = token_key(A, tok);
    const int32_t blk = A.tables[(int64_t)k.seq * A.max_blocks + k.block];
    const bool ok = in && blk >= 0 && blk < A.n_blocks;  // never write outside the pool
    const BlockRows B = block_rows(g, A.pool + (uint64_t)(ok ? blk : 0) * g.block_budget + (uint64_t)A.layer * g.layer_bytes, head, which);
    const float old_scale = k.slot > 0 && ok ? *B.scale : 0.f;
    float x[kEpl] = {};
    if (in) {
      rope::widen<kSrcF32>(w, x);
      if constexpr (ROPE != kPlain) {
        if (!which && L.live) rope::turn_row_at<ROPE, kSrcF32>(R, L, A.pos[tok], x, src, row);
      }
    }
    const float amax = row_max(amax8(0.f, x), lpr);
    const int e_old = k.slot > 0 ? stored_exponent(old_scale) : kScaleMin;
    const int e = max(e_old, scale_exponent(amax));
    if (ok) {
      if (k.slot > 0 && e > e_old) follow_scale(A, B.rows, k.slot, k.slot, e_old, e, lir, lpr);
      if (lir == 0) *B.scale = power_of_two(e);
      put_codes(A, B.rows, k.slot, L, split, x, power_of_two(-e));
    }
  }
}

// One append, dealt to n_teams teams of NWV waves; this one is number `team`.  A unit: the groups that begin among
// A.group_chunk neighbouring tokens, of them `heads` heads' K or V rows.  Groups of one token, a decode step's, are worked on side by side
// (16 384 of them 55 us; as groups like the others, one after the other, 385; prompts take the same with either, 125 and 123).
template <bool kSrcF32, int ROPE, int NWV, bool LATE, bool AHEAD>
__device__ __forceinline__ void append_groups(const AppendArgs& A, const rope::RopeArgs& R, int heads, int64_t team, int64_t n_teams, float* s_max,
                                              float* table) {
  const int lane = threadIdx.x & 63;
  const int parts = (A.g.H + heads - 1) / heads;
  const int64_t n_units = (A.n_tokens + A.group_chunk - 1) / A.group_chunk * (2 * parts);
  for (int64_t unit = team; unit < n_units; unit += n_teams) {
    int64_t chunk;
    int part;
    rope::split_unit(unit, (uint32_t)(2 * parts), chunk, part);
    const int which = part >= parts, h0 = (which ? part - parts : part) * heads, own_heads = min(heads, A.g.H - h0);
    chunk *= A.group_chunk;
    const rope::Lane L = block_lane<ROPE>(R, which, lane & ((1 << A.lpr_shift) - 1));
    const bool in = lane < A.group_chunk;
    const TokenKey own = token_key(A, in ? chunk + lane : -1), before = token_key(A, chunk + lane - 1);
    const bool leads = own.seq >= 0 && !(before.seq == own.seq && before.block == own.block);
    const TokenKey next = token_key(A, chunk + lane + 1);
    const bool alone = leads && !(next.seq == own.seq && next.block == own.block);
    const uint64_t singles = __ballot(alone);
    if (singles) append_singles<kSrcF32, ROPE, NWV>(A, R, L, chunk, singles, which, h0, own_heads);
    for (uint64_t leaders = __ballot(leads && !alone); leaders; leaders &= leaders - 1) {
      const int first = __builtin_ctzll(leaders);
      const Group G = find_group(A, chunk + first, __builtin_amdgcn_readlane(own.seq, first), __builtin_amdgcn_readlane(own.block, first));
      if (G.layer) append_group<kSrcF32, ROPE, NWV, LATE, AHEAD>(A, R, L, G, which, h0, own_heads, s_max, table);
    }
  }
}

// How a launch with one append works on it.
struct GroupPlan {
  int team;        // waves of a team: 4 or 8, a workgroup; or 1, four of them to a workgroup
  bool late;       // blocks hold more tokens than a team keeps
  int heads;       // heads of a unit
  int32_t chunk;   // AppendArgs::group_chunk
  int64_t blocks;  // workgroups
};

// BLOCK: the launch has FP8_BLOCK appends (kernels of their own: the groups take twice the registers of the rows).
template <bool kSrcF32, int HP, bool BLOCK>
__device__ __forceinline__ void append_any(const AppendArgs& A, int64_t worker, int64_t n_workers) {
  switch (A.g.dtype) {
    case FS_KV_FP16: append_rows<kSrcF32, FS_KV_FP16, HP>(A, worker, n_workers); break;
    case FS_KV_FP8_E4M3: append_rows<kSrcF32, FS_KV_FP8_E4M3, HP>(A, worker, n_workers); break;
    case FS_KV_INT8: append_rows<kSrcF32, FS_KV_INT8, HP>(A, worker, n_workers); break;
    case FS_KV_FP8_BLOCK:
      if constexpr (BLOCK) append_groups<kSrcF32, kPlain, 1, true, false>(A, rope::RopeArgs{}, 1, worker, n_workers, nullptr, nullptr);
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

append::GroupPlan plan_groups(const fs_pool* p, const append::AppendArgs& A);  // (fs_append.hip)

}  // namespace fs
