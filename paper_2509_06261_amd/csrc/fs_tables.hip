// fs_batch_tables: block tables, lengths, chunk offsets and token maps of a step from the requests' lengths, in one launch.
//
// FineServe Sec. 2.3 / 5.2: an engine keeps a block table per sequence and takes a block whenever a sequence crosses a block's
// end.  Which sequence a new token or block belongs to is a running sum over the requests.  A launch of its own for the sums
// would cost more than the sums: every workgroup works them out itself, a window of kWindow requests at a time, as far as its
// own share of the output, and looks its tokens (blocks) up in the window in LDS.
#include <algorithm>

#include "fs_internal.h"

namespace fs {
namespace {

constexpr int kThreads = 256, kPer = 4, kWindow = kThreads * kPer;
constexpr int kShare = 2048;  // tokens (or new blocks) of a workgroup

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
  uint32_t token_groups, id_groups;   // workgroups of the token maps, of the tables; behind them one for every window of requests
};

// A window's requests, and the sums up to it.
struct Window {
  int32_t held[kWindow], old_blocks[kWindow];
  int32_t token[kWindow + 1], block[kWindow + 1];  // the request's first new token, first new block (in the order of block_ids)
  int64_t sums[2][kThreads / 64];
};
struct Running {
  int64_t tokens = 0, blocks = 0;
  uint32_t flags = 0;
};

// x summed over the threads before this one, and `total` over all (every thread takes part).
__device__ __forceinline__ int64_t scan(int64_t x, int64_t* sums, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int64_t before = incl - x;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  return before;
}

// Lays window w out in LDS and adds it to the sums.
__device__ __forceinline__ void load_window(const TableArgs& A, int w, Window& W, Running& R) {
  __syncthreads();  // (the last window's readers are done)
  const int first = w * kWindow + (int)threadIdx.x * kPer;
  int32_t held[kPer], fresh[kPer];
  int64_t mine = 0;
  uint32_t flags = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = first + k;
    const int32_t h = b < A.n_seq && A.held ? A.held[b] : 0, n = b < A.n_seq ? A.fresh[b] : 0;
    held[k] = min(max(h, 0), A.cap);
    fresh[k] = min(max(n, 0), A.cap - held[k]);
    flags |= held[k] != h || fresh[k] != n;
    mine += fresh[k];
  }
  int64_t total;
  int64_t at = R.tokens + scan(mine, W.sums[0], total);
  R.tokens += total;
  int32_t need[kPer];
  mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {  // the new tokens that the lists have room for
    const int i = (int)threadIdx.x * kPer + k;
    const int32_t from = (int32_t)min(at, A.n_tokens);
    at += fresh[k];
    const int32_t n = (int32_t)min(at, A.n_tokens) - from;
    const int32_t old_blocks = (int32_t)(((uint32_t)held[k] + (uint32_t)A.T - 1) / (uint32_t)A.T);
    need[k] = (int32_t)(((uint32_t)held[k] + (uint32_t)n + (uint32_t)A.T - 1) / (uint32_t)A.T) - old_blocks;
    mine += need[k];
    W.held[i] = held[k];
    W.old_blocks[i] = old_blocks;
    W.token[i] = from;
  }
  int64_t block = R.blocks + scan(mine, W.sums[1], total);
  R.blocks += total;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    W.block[(int)threadIdx.x * kPer + k] = (int32_t)block;  // (no more new blocks than new tokens in the lists)
    block += need[k];
  }
  if (threadIdx.x == 0) {
    W.token[kWindow] = (int32_t)min(R.tokens, A.n_tokens);
    W.block[kWindow] = (int32_t)R.blocks;
  }
  if (__syncthreads_or(flags)) R.flags |= 1u;
  if (R.tokens > A.n_tokens || R.blocks > A.n_ids) R.flags |= 2u;
}

// The last request of the window whose first token (block) is at or before i.
__device__ __forceinline__ int owner(const int32_t (&first)[kWindow + 1], int32_t i) {
  int lo = 0;
#pragma unroll
  for (int step = kWindow / 2; step; step >>= 1)
    if (first[lo + step] <= i) lo += step;
  return lo;
}

__global__ __launch_bounds__(kThreads) void batch_tables_kernel(TableArgs A) {
  __shared__ Window W;
  const int windows = (A.n_seq + kWindow - 1) / kWindow;
  Running R;
  if (blockIdx.x < A.token_groups) {
    const int32_t lo = (int32_t)(blockIdx.x * (int64_t)kShare), hi = (int32_t)min((int64_t)lo + kShare, A.n_tokens);
    int32_t done = lo;  // tokens in front of it are written (uniform)
    for (int w = 0; w < windows && done < hi; ++w) {
      load_window(A, w, W, R);
      const int32_t end = min(hi, W.token[kWindow]);
      for (int32_t i = done + (int)threadIdx.x; i < end; i += kThreads) {
        const int k = owner(W.token, i), seq = w * kWindow + k;
        const int32_t p = W.held[k] + (i - W.token[k]);
        const int32_t b = (int32_t)((uint32_t)p / (uint32_t)A.T);
        A.seq_idx[i] = seq;
        A.pos[i] = p;
        if (A.slots) {
          int32_t id = -1;
          if (b < W.old_blocks[k]) {
            id = A.tables[(int64_t)seq * A.max_blocks + b];
          } else {
            const int64_t e = (int64_t)W.block[k] + (b - W.old_blocks[k]);
            if (e < A.n_ids) id = A.ids[e];
          }
          A.slots[i] = id >= 0 && id < A.n_blocks ? (int64_t)id * A.T + (p - b * A.T) : -1;
        }
      }
      done = max(done, end);
    }
    for (int32_t i = done + (int)threadIdx.x; i < hi; i += kThreads) {  // padding
      A.seq_idx[i] = -1;
      A.pos[i] = -1;
      if (A.slots) A.slots[i] = -1;
    }
  } else if (blockIdx.x < A.token_groups + A.id_groups) {
    // shares of the new blocks, until there are no more (more than block_ids has where that is too short)
    for (int64_t lo = (int64_t)(blockIdx.x - A.token_groups) * kShare;; lo += (int64_t)A.id_groups * kShare) {
      R = Running{};
      int64_t done = lo;
      for (int w = 0; w < windows && done < lo + kShare; ++w) {
        load_window(A, w, W, R);
        const int64_t end = min(lo + kShare, R.blocks);
        for (int64_t e = done + (int)threadIdx.x; e < end; e += kThreads) {
          const int k = owner(W.block, (int32_t)e);
          A.tables[(int64_t)(w * kWindow + k) * A.max_blocks + W.old_blocks[k] + (e - W.block[k])] = e < A.n_ids ? A.ids[e] : -1;
        }
        done = max(done, end);
      }
      if (done < lo + kShare) break;  // (uniform)
    }
  } else {
    const int own = (int)(blockIdx.x - A.token_groups - A.id_groups);
    for (int w = 0; w <= own; ++w) load_window(A, w, W, R);
    for (int k = threadIdx.x; k < kWindow && own * kWindow + k < A.n_seq; k += kThreads) {
      const int b = own * kWindow + k;
      A.seq_lens[b] = W.held[k] + (W.token[k + 1] - W.token[k]);
      A.q_offsets[b] = W.token[k];
    }
    if (own == windows - 1 && threadIdx.x == 0) {
      A.q_offsets[A.n_seq] = W.token[kWindow];
      if (A.status) *A.status = R.flags;
    }
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
  A.token_groups = (uint32_t)((n_tokens + kShare - 1) / kShare);
  A.id_groups = (uint32_t)std::max<int64_t>((n_block_ids + kShare - 1) / kShare, 1);
  const uint32_t windows = (uint32_t)((n_seq + kWindow - 1) / kWindow);
  (void)hipGetLastError();
  hipLaunchKernelGGL(batch_tables_kernel, dim3(A.token_groups + A.id_groups + windows), dim3(kThreads), 0, (hipStream_t)stream, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return device_error(e, "fs_batch_tables launch");
  return FS_OK;
}
