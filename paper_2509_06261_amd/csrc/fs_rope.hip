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
constexpr int kTurnRows = 4;  // rows of a unit in larger launches: the angles are worked out once for them (see wide_units)

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
// reads all of it before it writes: `out` may be `x`.  Bound by memory: 16 384 tokens of 32 heads of 128 in fp16, 268 MB read and written,
// 49 us, 5.5 TB/s (78 with the sines of every element by itself).
template <int MODE, bool kF32, bool kOutF32, int HP>
__global__ __launch_bounds__(kWaves * 64) void turn_kernel(TurnArgs A) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tpw = 64 >> A.lpr_shift;
  const Lane L = lane_of<MODE>(A.rope, lane & ((1 << A.lpr_shift) - 1));
  const Turns<MODE> turns = lane_turns<MODE>(A.rope, L);
  const uint32_t parts = (uint32_t)(A.n_heads + HP - 1) / HP;
  const int64_t n_units = (A.n_tokens + tpw - 1) / tpw * parts;
  for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < n_units; unit += (int64_t)gridDim.x * kWaves) {
    int64_t grp;
    int h0;
    split_unit(unit, parts, grp, h0);
    h0 *= HP;
    const int64_t tok = grp * tpw + (lane >> A.lpr_shift);
    const bool in = tok < A.n_tokens;
    auto row = [&](int k) { return tok * A.x_stride + (int64_t)(h0 + k) * A.d; };
    Raw<kF32> w[HP];
#pragma unroll
    for (int k = 0; k < HP; ++k)
      if (in && h0 + k < A.n_heads) load_raw<kF32, MODE == kSplit>(A.x, row(k), L, w[k]);
    const int pos = in ? A.pos[tok] : -1;  // (negative: padding, its row of out stays as it is)
    const Factors<MODE> F = factors<MODE>(A.rope, L, turns, max(pos, 0));
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      if (pos < 0 || h0 + k >= A.n_heads) continue;
      float x[kEpl];
      widen<kF32>(w[k], x);
      turn_row<MODE, kF32>(A.rope, L, F, x, A.x, row(k));
      store8<kOutF32, MODE == kSplit>(A.out, tok * A.out_stride + (int64_t)(h0 + k) * A.d, L, x);
    }
  }
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
template <int MODE, bool kSrcF32, int DT, int HP, bool CACHE>
__device__ __forceinline__ void rope_append_rows(const RopeAppendArgs& P, int64_t worker, int64_t n_workers) {
  const AppendArgs& A = P.a;
  const DevGeom& g = A.g;
  const int lane = threadIdx.x & 63;
  const int lpr = 1 << A.lpr_shift, tpw = 64 >> A.lpr_shift, lir = lane & (lpr - 1);
  const Lane L = lane_of<MODE>(P.rope, lir), plain{kEpl * lir, kEpl * lir + 4, 0, 0, false};
  const Turns<MODE> turns = lane_turns<MODE>(P.rope, L);
  const int rows = P.n_q + (CACHE ? 2 * g.H : 0), turned = P.n_q + (CACHE ? g.H : 0);
  const uint32_t parts = (uint32_t)(rows + HP - 1) / HP;
  const int64_t n_units = (A.n_tokens + tpw - 1) / tpw * parts;
  for (int64_t unit = worker; unit < n_units; unit += n_workers) {
    int64_t grp;
    int k0;
    split_unit(unit, parts, grp, k0);
    k0 *= HP;
    const int64_t tok = grp * tpw + (lane >> A.lpr_shift);
    const bool in = tok < A.n_tokens;
    auto source = [&](int r, const void*& src) {  // where row r begins (r is uniform)
      const bool is_q = r < P.n_q, is_k = r < turned;
      src = is_q ? P.q : is_k ? A.k_new : A.v_new;
      return tok * (is_q ? P.q_stride : is_k ? A.k_stride : A.v_stride) + (int64_t)(is_q ? r : is_k ? r - P.n_q : r - turned) * g.D;
    };
    Raw<kSrcF32> w[HP];
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      const int r = k0 + k;
      if (!in || r >= rows) continue;
      const void* src;
      const int64_t row = source(r, src);
      if (r < turned) load_raw<kSrcF32, MODE == kSplit>(src, row, L, w[k]);
      else load_raw<kSrcF32, false>(src, row, plain, w[k]);
    }
    const int pos = in ? A.pos[tok] : -1;
    Factors<MODE> F{};
    if (k0 < turned) F = factors<MODE>(P.rope, L, turns, max(pos, 0));
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
      float x[kEpl] = {};
      if (in) {
        widen<kSrcF32>(w[k], x);
        if (r < turned) {
          const void* src;
          const int64_t row = source(r, src);
          turn_row<MODE, kSrcF32>(P.rope, L, F, x, src, row);
        }
      }
      if (r < P.n_q) {
        if (pos >= 0) store8<false, MODE == kSplit>(P.q_out, (tok * P.n_q + r) * (int64_t)g.D, L, x);
      } else if constexpr (CACHE) {
        const int which = r >= turned, head = which ? r - turned : r - P.n_q;
        uint8_t* const chunk = layer + (uint64_t)head * g.head_chunk;
        uint8_t* const row = chunk + (which ? g.kv_tile : 0u) + (uint64_t)key.slot * g.row_bytes;
        uint8_t* const par = chunk + 2u * g.kv_tile + (which ? g.par_tile : 0u) + (uint64_t)key.slot * (uint32_t)g.param_bytes;
        const float sc = DT == FS_KV_FP8_E4M3 ? (which ? A.v_scale : A.k_scale)[head] : 1.0f;
        if (MODE == kSplit && !which) quantize_row<DT, true>(x, layer != nullptr, row, par, sc, lir, lpr, L.a, L.b);
        else quantize_row<DT>(x, layer != nullptr, row, par, sc, lir, lpr);
      }
    }
  }
}

template <int MODE, bool kSrcF32, int DT, int HP>
__global__ __launch_bounds__(kWaves * 64) void rope_append_kernel(RopeAppendArgs P) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  rope_append_rows<MODE, kSrcF32, DT, HP, true>(P, (int64_t)blockIdx.x * kWaves + wave, (int64_t)gridDim.x * kWaves);
}

// FP8_BLOCK: the keys and values by groups of a block's tokens (fs_append_block.h), the queries by rows.  The cache's workgroups
// come first: they take longest.  TEAM, heads: as in kv_append_block_kernel.  Dynamic LDS: the teams' tables of angles.
// Bound by the vector ALU (angles, rotation, conversion) and by memory about equally: four waves a SIMD, also where fp32 rows then spill some
// registers (65 600 tokens' keys and values, when this was chosen, 179 us and with three waves 186; with tokens of a group each beside them 198).
template <int MODE, bool kSrcF32, int TEAM, bool LATE, bool AHEAD>
__global__ __launch_bounds__((TEAM > 1 ? TEAM : kWaves) * 64, LATE ? 2 : 4) void rope_append_block_kernel(RopeAppendArgs P, int heads) {
  extern __shared__ float s_table[];
  constexpr int kOwn = TEAM > 1 ? TEAM : kWaves;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t cache_blocks = gridDim.x - P.q_blocks;
  if (blockIdx.x >= cache_blocks) {
    rope_append_rows<MODE, kSrcF32, FS_KV_FP8_BLOCK, 1, false>(P, (int64_t)(blockIdx.x - cache_blocks) * kOwn + wave, (int64_t)P.q_blocks * kOwn);
  } else if constexpr (TEAM == 1) {
    append_groups<kSrcF32, MODE, 1, LATE, AHEAD>(P.a, P.rope, heads, (int64_t)blockIdx.x * kWaves + wave, (int64_t)cache_blocks * kWaves, nullptr,
                                                   s_table + wave * table_floats(1));
  } else {
    __shared__ float s_max[2 * TEAM];
    append_groups<kSrcF32, MODE, TEAM, LATE, AHEAD>(P.a, P.rope, heads, blockIdx.x, cache_blocks, s_max, s_table);
  }
}

template <int MODE>
void (*turn_kernel_for(bool src_f32, bool out_f32, bool wide))(TurnArgs) {
  if (!src_f32) return wide ? turn_kernel<MODE, false, false, kTurnRows> : turn_kernel<MODE, false, false, 1>;
  if (out_f32) return wide ? turn_kernel<MODE, true, true, kTurnRows> : turn_kernel<MODE, true, true, 1>;
  return wide ? turn_kernel<MODE, true, false, kTurnRows> : turn_kernel<MODE, true, false, 1>;
}
template <int MODE, int DT>
void (*rope_append_kernel_of(bool f32, bool wide))(RopeAppendArgs) {
  if (f32) return wide ? rope_append_kernel<MODE, true, DT, kTurnRows> : rope_append_kernel<MODE, true, DT, 1>;
  return wide ? rope_append_kernel<MODE, false, DT, kTurnRows> : rope_append_kernel<MODE, false, DT, 1>;
}
template <int MODE>
void (*rope_append_kernel_for(int dtype, bool f32, bool wide))(RopeAppendArgs) {
  switch (dtype) {
    case FS_KV_FP16: return rope_append_kernel_of<MODE, FS_KV_FP16>(f32, wide);
    case FS_KV_FP8_E4M3: return rope_append_kernel_of<MODE, FS_KV_FP8_E4M3>(f32, wide);
    case FS_KV_INT8: return rope_append_kernel_of<MODE, FS_KV_INT8>(f32, wide);
    default: return rope_append_kernel_of<MODE, FS_KV_INT4>(f32, wide);
  }
}
template <int MODE, bool kF32>
void (*rope_append_block_kernel_for(const GroupPlan& G))(RopeAppendArgs, int) {
  // Rows ahead where a unit has several heads and the registers suffice.  (65 600 tokens' keys and values, 8 heads of 128, us without / with them:
  // fp16 in blocks of 63 137 / 125, of 128 174 / 166, of 16 148 / 138, and without a rotation 81 / 73, 108 / 95, 90 / 83; fp32 141 / 133 without a
  // rotation, but 198 / 261 with one.  With one head to a unit the kernel is the slower for them: a prompt of 777 tokens 12.5 / 14.)
  constexpr bool kAhead = !kF32 && MODE != kMixed;
#define FS_HEADS(TEAM) (kAhead && G.heads > 1 ? rope_append_block_kernel<MODE, kF32, TEAM, false, kAhead> : rope_append_block_kernel<MODE, kF32, TEAM, false, false>)
  return G.late ? rope_append_block_kernel<MODE, kF32, 8, true, false> : G.team == 8 ? FS_HEADS(8) : G.team == 4 ? FS_HEADS(4) : FS_HEADS(1);
#undef FS_HEADS
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

// Units of `hp` rows of `rows` each token has.
int64_t row_units(int64_t n_tokens, int lpr_shift, int rows, int hp) {
  const int64_t tpw = 64 >> lpr_shift;
  return (n_tokens + tpw - 1) / tpw * ((rows + hp - 1) / hp);
}

// Units of kTurnRows where there is one for every SIMD.  (us, single rows / four, units of four: queries of 4000 tokens, 32 heads of 128, 8000
// 16.6 / 12.0; of 1000, 2000 6.3 / 4.9; of 300, 600 4.2 / 4.2; with the rows of an FP16 cache 1000 tokens, 3000 8.8 / 7.2; 512, 1536 6.3 / 6.2;
// 300, 900 5.4 / 6.5.)
bool wide_units(const fs_pool* p, int64_t n_tokens, int lpr_shift, int rows) { return row_units(n_tokens, lpr_shift, rows, kTurnRows) >= (int64_t)p->n_cu * 4; }

hipError_t launch_turn(const fs_pool* p, const TurnArgs& A, bool src_f32, bool out_f32, hipStream_t s) {
  const bool wide = wide_units(p, A.n_tokens, A.lpr_shift, A.n_heads);
  const int64_t units = row_units(A.n_tokens, A.lpr_shift, A.n_heads, wide ? kTurnRows : 1);
  const unsigned blocks = (unsigned)std::min<int64_t>((units + kWaves - 1) / kWaves, (int64_t)p->n_cu * 64);
  const int mode = mode_of(A.rope);
  void (*const kern)(TurnArgs) = mode == kSplit   ? turn_kernel_for<kSplit>(src_f32, out_f32, wide)
                                 : mode == kPairs ? turn_kernel_for<kPairs>(src_f32, out_f32, wide)
                                                  : turn_kernel_for<kMixed>(src_f32, out_f32, wide);
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(kWaves * 64), 0, s, A);
  return hipGetLastError();
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
  if (M->rope_dim == 0) {
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
  (void)hipGetLastError();
  const hipError_t e = launch_turn(p, A, src_dtype == FS_SRC_FP32, src_dtype == FS_SRC_FP32, (hipStream_t)stream);
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
  if (M->rope_dim == 0) {
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
  const bool f32 = src_dtype == FS_SRC_FP32, block = M->g.kv_dtype == FS_KV_FP8_BLOCK;
  hipStream_t const s = (hipStream_t)stream;
  (void)hipGetLastError();
  hipError_t e = hipSuccess;
  const GroupPlan G = block ? plan_groups(p, P.a) : GroupPlan{};
  // FP8_BLOCK, many queries: they go in a launch of their own, whose waves take a third of the registers and four rows to a unit.  (us, one
  // launch / two, units of four: 64 000 tokens, 32 query heads of 128, 128 000 343 / 326; 8000, 16 000 51 / 44; 4000, 8000 35.2 / 32.9; 1000, 2000
  // 15.3 / 18.6.  The other formats' rows go with the queries': 64 000 tokens 285 / 299.)
  if (block && n_q_heads > 0 && row_units(n_tokens, P.a.lpr_shift, n_q_heads, kTurnRows) >= (int64_t)p->n_cu * 16) {
    TurnArgs T{};
    T.rope = P.rope;
    T.x = q;
    T.out = q_out;
    T.pos = pos;
    T.n_tokens = n_tokens;
    T.x_stride = q_stride;
    T.out_stride = q_row;
    T.n_heads = n_q_heads;
    T.d = d;
    T.lpr_shift = P.a.lpr_shift;
    e = launch_turn(p, T, f32, false, s);
    if (e != hipSuccess) return device_error(e, "fs_rope_append launch");
    P.n_q = 0;
  }
  const int64_t most = (int64_t)p->n_cu * 64;
  const int mode = mode_of(P.rope);
  if (block) {
    P.a.group_chunk = G.chunk;
    const int waves = G.team > 1 ? G.team : kWaves;
    if (P.n_q) P.q_blocks = (uint32_t)std::min((row_units(n_tokens, P.a.lpr_shift, P.n_q, 1) + waves - 1) / waves, most);
    const size_t lds = (size_t)table_floats(waves) * sizeof(float);  // (8 KB for every wave)
    void (*const kern)(RopeAppendArgs, int) =
        mode == kSplit   ? (f32 ? rope_append_block_kernel_for<kSplit, true>(G) : rope_append_block_kernel_for<kSplit, false>(G))
        : mode == kPairs ? (f32 ? rope_append_block_kernel_for<kPairs, true>(G) : rope_append_block_kernel_for<kPairs, false>(G))
                         : (f32 ? rope_append_block_kernel_for<kMixed, true>(G) : rope_append_block_kernel_for<kMixed, false>(G));
    hipLaunchKernelGGL(kern, dim3((unsigned)(G.blocks + P.q_blocks)), dim3(waves * 64), lds, s, P, G.heads);
  } else {
    const int rows = P.n_q + 2 * M->g.n_kv_heads;
    const bool wide = wide_units(p, n_tokens, P.a.lpr_shift, rows);
    const int64_t blocks = std::min((row_units(n_tokens, P.a.lpr_shift, rows, wide ? kTurnRows : 1) + kWaves - 1) / kWaves, most);
    const int dtype = M->g.kv_dtype;
    void (*const kern)(RopeAppendArgs) = mode == kSplit   ? rope_append_kernel_for<kSplit>(dtype, f32, wide)
                                         : mode == kPairs ? rope_append_kernel_for<kPairs>(dtype, f32, wide)
                                                          : rope_append_kernel_for<kMixed>(dtype, f32, wide);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kWaves * 64), 0, s, P);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return device_error(e, "fs_rope_append launch");
  return FS_OK;
}
