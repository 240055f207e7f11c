// Rotary positions: a model's rotation (fs_model_set_rope), rows by themselves (fs_rope), and a step's queries, keys and values
// on their way to the attention call and into the cache (fs_rope_append).
//
// FineServe Sec. 2.1: every new token appends its keys and values to the cache; models whose keys carry their position rotate
// them first.  Done here in the launch that appends, the keys are read once, rounded once (to the cache's format) and written
// once.  Everything below is bound by memory: a row is read and written once, and a wave works out the angles of its tokens once
// for several heads.
#include <algorithm>
#include <cmath>

#include "fs_append_block.h"

namespace fs {
namespace {

using namespace append;
using namespace rope;
constexpr int kWaves = 4;     // waves per workgroup
constexpr int kTurnRows = 4;  // rows of a unit in launches that leave every wave slot work, as kWideUnit

// ---- fs_rope ------------------------------------------------------------------------------------------------------
struct TurnArgs {
  RopeArgs rope;
  const void* x;
  void* out;
  const int32_t* pos;
  int64_t n_tokens, x_stride, out_stride;  // strides: elements from token to token
  int32_t n_heads, d, lpr_shift, pad;
};

// A unit: HP neighbouring heads of 64 / lpr consecutive tokens, a token's row per lpr lanes.  A row lies in one wave, which
// reads all of it before it writes: `out` may be `x`.
template <bool kF32, int HP>
__device__ __forceinline__ void turn_rows(const TurnArgs& A, int64_t worker, int64_t n_workers) {
  const int lane = threadIdx.x & 63;
  const int tpw = 64 >> A.lpr_shift, d0 = (lane & ((1 << A.lpr_shift) - 1)) * kEpl;
  const LaneTurns turns = lane_turns(A.rope, d0);
  const uint32_t parts = (uint32_t)(A.n_heads + HP - 1) / HP;
  const int64_t n_units = (A.n_tokens + tpw - 1) / tpw * parts;
  for (int64_t unit = worker; unit < n_units; unit += n_workers) {
    const int64_t grp = unit / parts;
    const int h0 = (int)(unit % parts) * HP;
    const int64_t tok = grp * tpw + (lane >> A.lpr_shift);
    const int pos = tok < A.n_tokens ? A.pos[tok] : -1;
    const bool ok = pos >= 0;  // (a negative position: padding, its row of out stays as it is)
    float x[HP][kEpl], y[HP][kEpl];
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      if (!ok || h0 + k >= A.n_heads) continue;
      const int64_t row = tok * A.x_stride + (int64_t)(h0 + k) * A.d;
      load8<kF32>(A.x, row + d0, x[k]);
      if (!A.rope.pairs && turns.live) load_partners<kF32>(A.x, row, turns, A.rope.dim, y[k]);
    }
    const Factors F = factors(A.rope, turns, max(pos, 0));
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      if (!ok || h0 + k >= A.n_heads) continue;
      if (turns.live) turn_row(A.rope, turns, F, x[k], y[k]);
      store8<kF32>(A.out, tok * A.out_stride + (int64_t)(h0 + k) * A.d + d0, x[k]);
    }
  }
}

template <bool kF32, int HP>
__global__ __launch_bounds__(kWaves * 64) void turn_kernel(TurnArgs A) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  turn_rows<kF32, HP>(A, (int64_t)blockIdx.x * kWaves + wave, (int64_t)gridDim.x * kWaves);
}

// ---- fs_rope_append -----------------------------------------------------------------------------------------------
struct RopeAppendArgs {
  AppendArgs a;
  RopeArgs rope;
  const void* q;
  void* q_out;  // fp16 [n_tokens][n_q][D]
  int64_t q_stride;
  int32_t n_q;
  uint32_t q_blocks;  // FP8_BLOCK: workgroups that work on the queries; the others work on the cache
};

// The place of a token's block in the cache (its layer), null if it has none.
__device__ __forceinline__ uint8_t* token_layer(const AppendArgs& A, const TokenKey& k) {
  if (k.seq < 0) return nullptr;
  const int32_t blk = A.tables[(int64_t)k.seq * A.max_blocks + k.block];
  if (blk < 0 || blk >= A.n_blocks) return nullptr;  // never write outside the pool
  return A.pool + (uint64_t)blk * A.g.block_budget + (uint64_t)A.layer * A.g.layer_bytes;
}

// Rows k0 .. k0 + HP - 1 of a token's n_q query heads, H key heads and H value heads.  CACHE = false: of its query heads alone.
template <bool kSrcF32, int DT, int HP, bool CACHE>
__device__ __forceinline__ void rope_append_rows(const RopeAppendArgs& P, int64_t worker, int64_t n_workers) {
  const AppendArgs& A = P.a;
  const DevGeom& g = A.g;
  const int lane = threadIdx.x & 63;
  const int lpr = 1 << A.lpr_shift, tpw = 64 >> A.lpr_shift, lir = lane & (lpr - 1), d0 = lir * kEpl;
  const LaneTurns turns = lane_turns(P.rope, d0);
  const int rows = P.n_q + (CACHE ? 2 * g.H : 0), turned = P.n_q + (CACHE ? g.H : 0);
  const uint32_t parts = (uint32_t)(rows + HP - 1) / HP;
  const int64_t n_units = (A.n_tokens + tpw - 1) / tpw * parts;
  for (int64_t unit = worker; unit < n_units; unit += n_workers) {
    const int64_t grp = unit / parts;
    const int k0 = (int)(unit % parts) * HP;
    const int64_t tok = grp * tpw + (lane >> A.lpr_shift);
    const bool in = tok < A.n_tokens;
    float x[HP][kEpl], y[HP][kEpl];
#pragma unroll
    for (int k = 0; k < HP; ++k) {
#pragma unroll
      for (int q = 0; q < kEpl; ++q) x[k][q] = y[k][q] = 0.f;
      const int r = k0 + k;  // (uniform)
      if (!in || r >= rows) continue;
      const bool is_q = r < P.n_q, is_k = !is_q && r < turned;
      const void* const src = is_q ? P.q : is_k ? A.k_new : A.v_new;
      const int head = is_q ? r : is_k ? r - P.n_q : r - turned;
      const int64_t row = tok * (is_q ? P.q_stride : is_k ? A.k_stride : A.v_stride) + (int64_t)head * g.D;
      load8<kSrcF32>(src, row + d0, x[k]);
      if (r < turned && !P.rope.pairs && turns.live) load_partners<kSrcF32>(src, row, turns, P.rope.dim, y[k]);
    }
    const int pos = in ? A.pos[tok] : -1;
    Factors F{};
    if (k0 < turned) F = factors(P.rope, turns, max(pos, 0));
    TokenKey key{-1, 0, 0};
    uint8_t* layer = nullptr;
    if (CACHE && k0 + HP > P.n_q) {
      key = token_key(A, tok);
      layer = token_layer(A, key);
    }
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      const int r = k0 + k;
      if (r >= rows) break;
      if (r < turned && turns.live) turn_row(P.rope, turns, F, x[k], y[k]);
      if (r < P.n_q) {
        if (pos >= 0) store8<false>(P.q_out, (tok * P.n_q + r) * (int64_t)g.D + d0, x[k]);
      } else if constexpr (CACHE) {
        const int which = r >= turned, head = which ? r - turned : r - P.n_q;
        uint8_t* const chunk = layer + (uint64_t)head * g.head_chunk;
        uint8_t* const row = chunk + (which ? g.kv_tile : 0u) + (uint64_t)key.slot * g.row_bytes;
        uint8_t* const par = chunk + 2u * g.kv_tile + (which ? g.par_tile : 0u) + (uint64_t)key.slot * (uint32_t)g.param_bytes;
        const float sc = DT == FS_KV_FP8_E4M3 ? (which ? A.v_scale : A.k_scale)[head] : 1.0f;
        quantize_row<DT>(x[k], layer != nullptr, row, par, sc, lir, lpr);
      }
    }
  }
}

template <bool kSrcF32, int DT, int HP>
__global__ __launch_bounds__(kWaves * 64) void rope_append_kernel(RopeAppendArgs P) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  rope_append_rows<kSrcF32, DT, HP, true>(P, (int64_t)blockIdx.x * kWaves + wave, (int64_t)gridDim.x * kWaves);
}

// FP8_BLOCK: the keys and values by groups of a block's tokens (fs_append_block.h), the queries by rows.
template <bool kSrcF32, int HP>
__global__ __launch_bounds__(kWaves * 64) void rope_append_block_kernel(RopeAppendArgs P) {
  __shared__ float s_max[kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x < P.q_blocks)
    rope_append_rows<kSrcF32, FS_KV_FP8_BLOCK, HP, false>(P, (int64_t)blockIdx.x * kWaves + wave, (int64_t)P.q_blocks * kWaves);
  else
    append_groups<kSrcF32, true, kWaves>(P.a, P.rope, blockIdx.x - P.q_blocks, gridDim.x - P.q_blocks, s_max);
}

RopeArgs rope_args(const Model& M, int inverse) {
  RopeArgs R{};
  R.turns = M.d_turns;
  R.dim = M.rope_dim;
  R.pairs = M.rope_layout == FS_ROPE_PAIRS;
  R.amplitude = M.rope_amplitude;
  R.direction = inverse ? -1.0f : 1.0f;
  return R;
}

int lanes_shift(int head_dim) {
  int s = 0;
  while ((kEpl << s) < head_dim) ++s;
  return s;
}

// Radians per position of every pair, or false for parameters that make none.
bool frequencies(const fs_rope_t& r, long double* f) {
  const long double pi2 = 6.283185307179586476925286766559L;
  auto good = [](double x) { return x > 0.0 && x < 1e300; };
  if (r.rotary_dim < 2 || (r.rotary_dim & 1) || r.rotary_dim > 512 || (r.layout != FS_ROPE_HALVES && r.layout != FS_ROPE_PAIRS) ||
      !(r.base > 1.0) || !good(r.base) || !good(r.amplitude) || r.scaling < FS_ROPE_UNSCALED || r.scaling > FS_ROPE_DIMENSION)
    return false;
  if (r.scaling != FS_ROPE_UNSCALED && !good(r.factor)) return false;
  if (r.scaling == FS_ROPE_BASE && r.rotary_dim < 4) return false;
  if (r.scaling >= FS_ROPE_WAVELENGTH &&
      (r.original_positions < 1 || !(r.low >= 0.0) || !(r.high > r.low) || !good(r.high) || (r.scaling == FS_ROPE_DIMENSION && !(r.low > 0.0))))
    return false;
  const long double dim = r.rotary_dim, factor = r.factor, orig = r.original_positions;
  long double base = r.base;
  if (r.scaling == FS_ROPE_BASE) base *= powl(factor, dim / (dim - 2));
  long double first = 0, last = 0;
  if (r.scaling == FS_ROPE_DIMENSION) {
    auto at = [&](long double turns) { return dim * logl(orig / (turns * pi2)) / (2 * logl(base)); };
    first = std::max(floorl(at(r.high)), 0.0L);
    last = std::min(ceill(at(r.low)), dim - 1);
  }
  for (int i = 0; i < r.rotary_dim / 2; ++i) {
    long double x = powl(base, -2.0L * i / dim), stretch = 0;  // stretch: how much of the factor the pair takes, 0 .. 1
    if (r.scaling == FS_ROPE_LINEAR) stretch = 1;
    if (r.scaling == FS_ROPE_WAVELENGTH) stretch = 1 - std::min(std::max((orig * x / pi2 - r.low) / (r.high - r.low), 0.0L), 1.0L);
    if (r.scaling == FS_ROPE_DIMENSION) stretch = std::min(std::max((i - first) / std::max(last - first, 0.001L), 0.0L), 1.0L);
    if (stretch > 0) x = x * (1 - stretch) + x / factor * stretch;
    f[i] = x;
  }
  return true;
}

Model* rope_model(fs_pool* p, fs_model_t model, const char* who) {
  if (!p || model < 0 || model >= kMaxModels || !p->models[model].in_use) {
    set_error(std::string(who) + ": unknown model");
    return nullptr;
  }
  return &p->models[model];
}

}  // namespace
}  // namespace fs

using namespace fs;

extern "C" int fs_rope_frequencies(const fs_rope_t* rope, double* radians) {
  long double f[256];
  if (!rope || !radians || !frequencies(*rope, f)) {
    set_error("fs_rope_frequencies: invalid argument");
    return FS_ERR_INVALID;
  }
  for (int i = 0; i < rope->rotary_dim / 2; ++i) radians[i] = (double)f[i];
  return FS_OK;
}

extern "C" int fs_model_set_rope(fs_pool* p, fs_model_t model, const fs_rope_t* rope) {
  Model* M = rope_model(p, model, "fs_model_set_rope");
  if (!M) return FS_ERR_INVALID;
  long double f[256];
  if (!rope || rope->rotary_dim > M->g.head_dim || !frequencies(*rope, f)) {
    set_error("fs_model_set_rope: invalid rotation");
    return FS_ERR_INVALID;
  }
  if (p->n_cu == 0) {
    set_error("fs_model_set_rope: pool has no HIP device");
    return FS_ERR_DEVICE;
  }
  uint64_t turns[256];
  for (int i = 0; i < rope->rotary_dim / 2; ++i) {
    // turns per position, less whole ones, as a fraction of 2^64 (long double's 64 bits hold it)
    const long double t = fmodl(f[i] / 6.283185307179586476925286766559L, 1.0L) * 18446744073709551616.0L;
    turns[i] = t >= 18446744073709551615.0L ? ~0ull : (uint64_t)t;
  }
  hipError_t e;
  if (!M->d_turns && (e = hipMalloc((void**)&M->d_turns, (size_t)M->g.head_dim / 2 * sizeof(uint64_t))) != hipSuccess)
    return device_error(e, "hipMalloc");
  if ((e = hipMemcpy(M->d_turns, turns, (size_t)rope->rotary_dim / 2 * sizeof(uint64_t), hipMemcpyHostToDevice)) != hipSuccess)
    return device_error(e, "hipMemcpy(rope)");
  M->rope_dim = rope->rotary_dim;
  M->rope_layout = rope->layout;
  M->rope_amplitude = (float)rope->amplitude;
  return FS_OK;
}

extern "C" int fs_rope(fs_pool* p, fs_model_t model, const void* x, int64_t x_stride, int n_heads, int src_dtype, const int32_t* pos,
                       int64_t n_tokens, int inverse, void* out, int64_t out_stride, void* stream) {
  const Model* M = rope_model(p, model, "fs_rope");
  if (!M) return FS_ERR_INVALID;
  const int d = M->g.head_dim, per = src_dtype == FS_SRC_FP32 ? 4 : 8;  // elements in 16 bytes
  if (n_tokens < 0 || n_heads < 1 || n_heads > 65536 || (src_dtype != FS_SRC_FP16 && src_dtype != FS_SRC_FP32) ||
      (n_tokens > 0 && (!x || !pos || !out))) {
    set_error("fs_rope: invalid argument");
    return FS_ERR_INVALID;
  }
  const int64_t row = (int64_t)n_heads * d;
  if (x_stride == 0) x_stride = row;
  if (out_stride == 0) out_stride = row;
  if (x_stride < row || out_stride < row || ((x_stride | out_stride) % per) || (((uintptr_t)x | (uintptr_t)out) & 15)) {
    set_error("fs_rope: rows must not overlap and must be 16-byte aligned");
    return FS_ERR_INVALID;
  }
  if (!M->d_turns) {
    set_error("fs_rope: the model has no rotation (fs_model_set_rope)");
    return FS_ERR_INVALID;
  }
  if (n_tokens == 0) return FS_OK;
  TurnArgs A{};
  A.rope = rope_args(*M, inverse);
  A.x = x;
  A.out = out;
  A.pos = pos;
  A.n_tokens = n_tokens;
  A.x_stride = x_stride;
  A.out_stride = out_stride;
  A.n_heads = n_heads;
  A.d = d;
  A.lpr_shift = lanes_shift(d);
  const int64_t tpw = 64 >> A.lpr_shift, groups = (n_tokens + tpw - 1) / tpw;
  const bool wide = groups * ((n_heads + kTurnRows - 1) / kTurnRows) >= (int64_t)p->n_cu * 32;
  const int64_t units = groups * (wide ? (n_heads + kTurnRows - 1) / kTurnRows : n_heads);
  const unsigned blocks = (unsigned)std::min<int64_t>((units + kWaves - 1) / kWaves, (int64_t)p->n_cu * 64);
  void (*const kern)(TurnArgs) = src_dtype == FS_SRC_FP32 ? (wide ? turn_kernel<true, kTurnRows> : turn_kernel<true, 1>)
                                                          : (wide ? turn_kernel<false, kTurnRows> : turn_kernel<false, 1>);
  (void)hipGetLastError();
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(kWaves * 64), 0, (hipStream_t)stream, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return device_error(e, "fs_rope launch");
  return FS_OK;
}

extern "C" int fs_rope_append(fs_pool* p, fs_model_t model, int layer, const void* q, int64_t q_stride, int n_q_heads, const void* k,
                              int64_t k_stride, const void* v, int64_t v_stride, int src_dtype, const int32_t* seq_idx,
                              const int32_t* pos, const int32_t* block_tables, int max_blocks, int64_t n_tokens, void* q_out,
                              void* stream) {
  const Model* M = rope_model(p, model, "fs_rope_append");
  if (!M) return FS_ERR_INVALID;
  const int d = M->g.head_dim, per = src_dtype == FS_SRC_FP32 ? 4 : 8;
  if (n_q_heads < 0 || n_q_heads > 65536 || (n_q_heads > 0 && n_tokens > 0 && (!q || !q_out))) {
    set_error("fs_rope_append: invalid argument");
    return FS_ERR_INVALID;
  }
  const int64_t q_row = (int64_t)n_q_heads * d, kv_row = (int64_t)M->g.n_kv_heads * d;
  if (q_stride == 0) q_stride = q_row;
  if (k_stride == 0) k_stride = kv_row;
  if (v_stride == 0) v_stride = kv_row;
  if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row || ((q_stride | k_stride | v_stride) % per) ||
      (n_q_heads > 0 && (((uintptr_t)q | (uintptr_t)q_out) & 15))) {
    set_error("fs_rope_append: rows must not overlap and must be 16-byte aligned");
    return FS_ERR_INVALID;
  }
  fs_append_t a{};
  a.model = model;
  a.layer = layer;
  a.src_dtype = src_dtype;
  a.max_blocks = max_blocks;
  a.k_new = k;
  a.v_new = v;
  a.seq_idx = seq_idx;
  a.pos = pos;
  a.block_tables = block_tables;
  a.n_tokens = n_tokens;
  RopeAppendArgs P{};
  const int rc = make_append_args(p, a, P.a);
  if (rc != FS_OK) return rc;
  if (!M->d_turns) {
    set_error("fs_rope_append: the model has no rotation (fs_model_set_rope)");
    return FS_ERR_INVALID;
  }
  if (n_tokens == 0) return FS_OK;
  P.rope = rope_args(*M, 0);
  P.q = q;
  P.q_out = q_out;
  P.q_stride = q_stride;
  P.n_q = n_q_heads;
  P.a.k_stride = k_stride;
  P.a.v_stride = v_stride;
  const int64_t tpw = 64 >> P.a.lpr_shift, groups = (n_tokens + tpw - 1) / tpw, most = (int64_t)p->n_cu * 64;
  const bool block = M->g.kv_dtype == FS_KV_FP8_BLOCK;
  const int rows = n_q_heads + (block ? 0 : 2 * M->g.n_kv_heads);
  const bool wide = groups * ((rows + kTurnRows - 1) / kTurnRows) >= (int64_t)p->n_cu * 32;
  const int64_t units = groups * (wide ? (rows + kTurnRows - 1) / kTurnRows : rows);
  int64_t blocks = std::min((units + kWaves - 1) / kWaves, most);
  const bool f32 = src_dtype == FS_SRC_FP32;
  void (*kern)(RopeAppendArgs) = nullptr;
  if (block) {
    P.q_blocks = (uint32_t)blocks;
    P.a.group_chunk = group_chunk(n_tokens, 2 * M->g.n_kv_heads, (int64_t)p->n_cu * 8);
    blocks += std::min((n_tokens + P.a.group_chunk - 1) / P.a.group_chunk * 2 * M->g.n_kv_heads, most);
    kern = f32 ? (wide ? rope_append_block_kernel<true, kTurnRows> : rope_append_block_kernel<true, 1>)
               : (wide ? rope_append_block_kernel<false, kTurnRows> : rope_append_block_kernel<false, 1>);
  } else {
#define FS_ROPE_APPEND(DT)                                                                                  \
  (f32 ? (wide ? rope_append_kernel<true, DT, kTurnRows> : rope_append_kernel<true, DT, 1>)                 \
       : (wide ? rope_append_kernel<false, DT, kTurnRows> : rope_append_kernel<false, DT, 1>))
    switch (M->g.kv_dtype) {
      case FS_KV_FP16: kern = FS_ROPE_APPEND(FS_KV_FP16); break;
      case FS_KV_FP8_E4M3: kern = FS_ROPE_APPEND(FS_KV_FP8_E4M3); break;
      case FS_KV_INT8: kern = FS_ROPE_APPEND(FS_KV_INT8); break;
      default: kern = FS_ROPE_APPEND(FS_KV_INT4); break;
    }
#undef FS_ROPE_APPEND
  }
  (void)hipGetLastError();
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kWaves * 64), 0, (hipStream_t)stream, P);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return device_error(e, "fs_rope_append launch");
  return FS_OK;
}
