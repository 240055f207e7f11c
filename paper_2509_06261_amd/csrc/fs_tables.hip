// fs_batch_tables: block tables, lengths, chunk offsets and token maps of a step from the requests' lengths, in one launch.
//
// FineServe Sec. 2.3 / 5.2: an engine keeps a block table per sequence and takes a block whenever a sequence crosses a block's
// end.  Where a request's tokens and blocks begin is a sum over the requests in front of it.  A launch of its own for the sums
// would cost more than they do: every workgroup adds all requests up for itself (8 bytes each, from the L2), which also tells it
// where the padding begins, and then writes what belongs to its own few requests -- nothing has to be searched.
// (2048 prompts of up to 900 tokens, 15 MB written: 17 us with running sums over windows of 1024 requests in LDS and a search for
// every token's request, 12.9 with this, of which the writes are 3; 20 000 requests of up to 40 tokens 86 -> 34.  The smallest calls, the
// newest tokens of eight requests, take 4.2 us, a launch.)
#include <algorithm>

#include "fs_internal.h"

namespace fs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct TableArgs {
  const int32_t* held;
  const int32_t* fresh;
  const int32_t* ids;
  int32_t* tables;
  int32_t* seq_lens;
  int32_t* q_offsets;
  int32_t* seq_idx;
  int32_t* pos;
  int64_t* slots;
  uint32_t* status;
  int64_t n_ids, n_tokens, n_blocks;
  int32_t n_seq, max_blocks, T, cap;  // cap: tokens that a table's row has blocks for
  uint32_t t_magic, t_shift;          // (see over_t: the shift less one)
  int32_t group, parts;               // requests of a workgroup (up to 64), workgroups that share them
};

// A request's lengths, within what its table can hold.
struct Request {
  int32_t held, fresh;
  bool clamped;
};
__device__ __forceinline__ Request request(const TableArgs& A, int b) {
  const int32_t h = A.held ? A.held[b] : 0, n = A.fresh[b];
  Request r;
  r.held = min(max(h, 0), A.cap);
  r.fresh = min(max(n, 0), A.cap - r.held);
  r.clamped = r.held != h || r.fresh != n;
  return r;
}
// x / T for 0 <= x < 2^31: with 2^s >= T the factor m = ceil(2^(31 + s) / T) fits 32 bits, and x m / 2^(31 + s) exceeds x / T by less
// than 2^s x / (2^(31 + s) T) < 1 / T.
__device__ __forceinline__ int32_t over_t(const TableArgs& A, int32_t x) {
  return A.T == 1 ? x : (int32_t)(__umulhi((uint32_t)x, A.t_magic) >> A.t_shift);
}
__device__ __forceinline__ int32_t blocks_of(const TableArgs& A, int32_t tokens) { return tokens ? over_t(A, tokens - 1) + 1 : 0; }

struct Sums {
  int64_t tokens, blocks, tokens_before, blocks_before;  // new ones: of all requests, of those in front of the workgroup's first
  int32_t clamped;
};
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ Sums add_up(const TableArgs& A, int first, Sums* s_waves) {
  Sums s{0, 0, 0, 0, 0};
#pragma unroll 4
  for (int b = threadIdx.x; b < A.n_seq; b += kThreads) {
    const Request r = request(A, b);
    const int32_t need = blocks_of(A, r.held + r.fresh) - blocks_of(A, r.held);
    s.tokens += r.fresh;
    s.blocks += need;
    s.tokens_before += b < first ? r.fresh : 0;
    s.blocks_before += b < first ? need : 0;
    s.clamped |= r.clamped;
  }
  s.tokens = wave_sum(s.tokens);
  s.blocks = wave_sum(s.blocks);
  s.tokens_before = wave_sum(s.tokens_before);
  s.blocks_before = wave_sum(s.blocks_before);
  s.clamped = __any(s.clamped);
  if ((threadIdx.x & 63) == 0) s_waves[threadIdx.x >> 6] = s;
  __syncthreads();
  s = s_waves[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    s.tokens += s_waves[w].tokens;
    s.blocks += s_waves[w].blocks;
    s.tokens_before += s_waves[w].tokens_before;
    s.blocks_before += s_waves[w].blocks_before;
    s.clamped |= s_waves[w].clamped;
  }
  return s;
}
// x summed over the lanes before this one.
__device__ __forceinline__ int64_t lanes_before(int64_t x) {
  const int lane = threadIdx.x & 63;
  int64_t incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  return incl - x;
}

// Workgroup (group, part): requests group * A.group .., every A.parts-th share of their tokens and blocks.
__global__ __launch_bounds__(kThreads) void batch_tables_kernel(TableArgs A) {
  __shared__ Sums s_waves[kWaves];
  const int part = blockIdx.x % A.parts, first = (int)(blockIdx.x / A.parts) * A.group;
  const Sums all = add_up(A, first, s_waves);
  // Lane l of every wave: request first + l, and where its tokens and blocks begin.  Tokens that the lists have no room for are
  // cut, and with them the blocks that only they need.  (Behind a cut nothing begins, so that it does not matter that the blocks in
  // front of this group were counted without one.)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = first + lane, n_own = min(A.group, A.n_seq - first);
  Request r{0, 0, false};
  if (lane < n_own) r = request(A, b);
  const int64_t at = all.tokens_before + lanes_before(r.fresh);
  const int32_t token = (int32_t)min(at, A.n_tokens), fresh = (int32_t)min(at + r.fresh, A.n_tokens) - token;
  const int32_t old_blocks = blocks_of(A, r.held), need = blocks_of(A, r.held + fresh) - old_blocks;
  const int32_t block = (int32_t)min(all.blocks_before + lanes_before(need), (int64_t)0x7fffffff);
  if (part == 0 && wave == 0 && lane < n_own) {
    A.seq_lens[b] = r.held + fresh;
    A.q_offsets[b] = token;
    if (b == A.n_seq - 1) A.q_offsets[A.n_seq] = token + fresh;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && A.status)
    *A.status = (all.clamped ? 1u : 0u) | (all.tokens > A.n_tokens || all.blocks > A.n_ids ? 2u : 0u);
  // a request's tokens go to the waves of its parts in turn, another wave first for every request
  const int units = A.parts * kWaves, unit = part * kWaves + wave, stride = units * 64;
  for (int k = 0; k < n_own; ++k) {
    const int turn = unit >= k % units ? unit - k % units : unit + units - k % units;
    const int32_t n = __builtin_amdgcn_readlane(fresh, k);
    if (turn * 64 >= n) continue;  // (uniform; there are no more blocks than tokens)
    const int32_t held = __builtin_amdgcn_readlane(r.held, k), to = __builtin_amdgcn_readlane(token, k), old = __builtin_amdgcn_readlane(old_blocks, k),
                  more = __builtin_amdgcn_readlane(need, k), from = __builtin_amdgcn_readlane(block, k);
    int32_t* const row = A.tables + (int64_t)(first + k) * A.max_blocks;
    for (int32_t e = turn * 64 + lane; e < more; e += stride) row[old + e] = (int64_t)from + e < A.n_ids ? A.ids[from + e] : -1;
#pragma unroll 2
    for (int32_t j = turn * 64 + lane; j < n; j += stride) {
      const int32_t p = held + j, i = to + j;
      A.seq_idx[i] = first + k;
      A.pos[i] = p;
      if (A.slots) {
        const int32_t q = over_t(A, p);
        int32_t id = -1;
        if (q < old) id = row[q];  // (not written by this launch)
        else if ((int64_t)from + (q - old) < A.n_ids) id = A.ids[from + (q - old)];
        A.slots[i] = id >= 0 && id < A.n_blocks ? (int64_t)id * A.T + (p - q * A.T) : -1;
      }
    }
  }
  for (int64_t i = min(all.tokens, A.n_tokens) + (int64_t)blockIdx.x * kThreads + threadIdx.x; i < A.n_tokens; i += (int64_t)gridDim.x * kThreads) {
    A.seq_idx[i] = -1;  // padding
    A.pos[i] = -1;
    if (A.slots) A.slots[i] = -1;
  }
}

}  // namespace
}  // namespace fs

using namespace fs;

extern "C" int fs_batch_tables(fs_pool* p, fs_model_t model, const int32_t* held_lens, const int32_t* new_lens, int n_seq,
                               const int32_t* block_ids, int64_t n_block_ids, int32_t* block_tables, int max_blocks, int32_t* seq_lens,
                               int32_t* q_offsets, int32_t* seq_idx, int32_t* pos, int64_t* slots, int64_t n_tokens, uint32_t* status,
                               void* stream) {
  if (!p || model < 0 || model >= kMaxModels || !p->models[model].in_use) {
    set_error("fs_batch_tables: unknown model");
    return FS_ERR_INVALID;
  }
  if (n_seq < 1 || max_blocks < 1 || !new_lens || !block_tables || !seq_lens || !q_offsets || n_block_ids < 0 ||
      (n_block_ids > 0 && !block_ids) || n_tokens < 0 || n_tokens > 0x7fffffff || (n_tokens > 0 && (!seq_idx || !pos))) {
    set_error("fs_batch_tables: invalid argument");
    return FS_ERR_INVALID;
  }
  if (n_seq > 0x3fffffff || n_block_ids > 0x7fffffff) {
    set_error("fs_batch_tables: batch too large");
    return FS_ERR_INVALID;
  }
  if (p->n_cu == 0) {
    set_error("fs_batch_tables: pool has no HIP device");
    return FS_ERR_DEVICE;
  }
  const fs_geometry_t& g = p->models[model].g;
  TableArgs A{};
  A.held = held_lens;
  A.fresh = new_lens;
  A.ids = block_ids;
  A.tables = block_tables;
  A.seq_lens = seq_lens;
  A.q_offsets = q_offsets;
  A.seq_idx = seq_idx;
  A.pos = pos;
  A.slots = slots;
  A.status = status;
  A.n_ids = n_block_ids;
  A.n_tokens = n_tokens;
  A.n_blocks = (int64_t)(p->pool_bytes / g.block_budget);
  A.n_seq = n_seq;
  A.max_blocks = max_blocks;
  A.T = g.tokens_per_block;
  A.cap = (int32_t)std::min<int64_t>((int64_t)max_blocks * g.tokens_per_block, 0x7fffffff);
  int shift = 0;
  while ((1ll << shift) < A.T) ++shift;
  A.t_magic = A.T == 1 ? 0u : (uint32_t)(((1ull << (31 + shift)) + (uint64_t)A.T - 1) / (uint64_t)A.T);
  A.t_shift = shift ? (uint32_t)shift - 1 : 0u;
  // One workgroup per compute unit, up to four where there are more than four turns of its threads to write; requests are shared where
  // they are fewer.  (All of them add all requests up: the newest tokens of 3000 requests 10.7 us with four per unit.)
  const int64_t wgs = std::min<int64_t>(std::max<int64_t>(p->n_cu, n_tokens / (4 * kThreads)), (int64_t)p->n_cu * 4);
  A.group = (int32_t)std::min<int64_t>((n_seq + wgs - 1) / wgs, 64);
  const int64_t groups = (n_seq + A.group - 1) / A.group;
  A.parts = (int32_t)std::max<int64_t>(std::min<int64_t>(n_tokens / (groups * 4 * kThreads), wgs / groups), 1);
  (void)hipGetLastError();
  hipLaunchKernelGGL(batch_tables_kernel, dim3((unsigned)(groups * A.parts)), dim3(kThreads), 0, (hipStream_t)stream, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return device_error(e, "fs_batch_tables launch");
  return FS_OK;
}
