// The accepted path of a tree of drafts joins the cache (what pe_append_kv does for one token of every sequence): copies, bound by
// memory, or for small batches by the launch (3.3 to 3.9 us for 8 sequences; for 256 sequences with eight heads of D = 128, up to a page's 16
// tokens of each, 6 to 7).
//
// One workgroup per sequence takes what is left of the sequence's path up to the end of its newest page: lengths and progress are
// read and written by that workgroup alone, so both are updated in place.  Phase 1 links a new page into each row when the newest
// one is full; phase 2 copies token rows, 16 bytes a lane.
#include "pe_device.h"
#include "pe_rows.h"

namespace pe {
namespace {

constexpr int kThreads = kPathThreads;
constexpr int kMostTokens = 128;  // of a page

__global__ __launch_bounds__(kThreads) void append_path_kernel(const uint4* __restrict__ k_draft, const uint4* __restrict__ v_draft,
                                                               const int32_t* __restrict__ path, const int32_t* __restrict__ path_lens,
                                                               int32_t* __restrict__ path_done, uint4* __restrict__ k_pool,
                                                               uint4* __restrict__ v_pool, int32_t* __restrict__ block_table,
                                                               int32_t* __restrict__ seq_lens, int32_t* __restrict__ freed_phys,
                                                               const int32_t* __restrict__ spare, int32_t* __restrict__ spare_used,
                                                               int n_spare, int drafts, int max_path, int rows_per_seq, int block_size,
                                                               int max_blocks, int vec_per_row) {
  __shared__ int32_t draft_of[kMostTokens];
  __shared__ int bad;
  const int s = (int)blockIdx.x, me = (int)threadIdx.x;
  const int len = seq_lens[s], done = path_done[s], have = path_lens[s];
  const int slot = len % block_size, jb = len / block_size;
  const int end = have < max_path ? have : max_path;
  if (len < 0 || jb >= max_blocks || done < 0 || done >= end) return;  // nothing left, or a caller precondition violated: all untouched
  int count = end - done < block_size - slot ? end - done : block_size - slot;
  if (me == 0) bad = count;
  __syncthreads();
  if (me < count) {
    const int d = path[(int64_t)s * max_path + done + me];
    draft_of[me] = d;
    if (d < 0 || d >= drafts) atomicMin(&bad, me);  // the path ends in front of what is no draft
  }
  __syncthreads();
  count = bad;
  if (count == 0) return;
  if (slot == 0) {
    for (int h = me; h < rows_per_seq; h += kThreads) {
      const int64_t row = (int64_t)s * rows_per_seq + h;
      int32_t page = freed_phys[row];
      if (page >= 0) {
        freed_phys[row] = -1;
      } else {
        const int used = spare_used[row];
        page = used >= 0 && used < n_spare ? spare[row * n_spare + used] : -1;
        spare_used[row] = used + 1;
      }
      block_table[row * max_blocks + jb] = page;
    }
  }
  __syncthreads();
  const int per_token = rows_per_seq * vec_per_row, all = count * per_token;
  const int64_t from = (int64_t)s * drafts * per_token;
  for (int idx = me; idx < all; idx += kThreads) {
    const int i = idx / per_token, rest = idx - i * per_token, h = rest / vec_per_row, u = rest - h * vec_per_row;
    const int32_t page = block_table[((int64_t)s * rows_per_seq + h) * max_blocks + jb];
    if (page < 0) continue;  // spare list exhausted (precondition violated): the tokens are dropped
    const int64_t to = ((int64_t)page * block_size + slot + i) * vec_per_row + u;
    const int64_t src = from + (int64_t)draft_of[i] * per_token + rest;
    k_pool[to] = k_draft[src];
    v_pool[to] = v_draft[src];
  }
  if (me == 0) {
    seq_lens[s] = len + count;
    path_done[s] = done + count;
  }
}

}  // namespace

hipError_t launch_append_path(const PathArgs& a, hipStream_t stream) {
  const int vec_per_head_row = a.head_dim * (a.is_bf16 ? 2 : 4) / 16;
  const int rows_per_seq = a.shared ? 1 : a.num_kv_heads;
  const int vec_per_row = a.shared ? vec_per_head_row * a.num_kv_heads : vec_per_head_row;
  hipLaunchKernelGGL(append_path_kernel, dim3((unsigned)a.num_seqs), dim3(kThreads), 0, stream, (const uint4*)a.k_draft,
                     (const uint4*)a.v_draft, a.path, a.path_lens, a.path_done, (uint4*)a.k_pool, (uint4*)a.v_pool, a.block_table,
                     a.seq_lens, a.freed_phys, a.spare, a.spare_used, a.n_spare, a.drafts, a.max_path, rows_per_seq, a.block_size,
                     a.max_blocks, vec_per_row);
  return hipGetLastError();
}

}  // namespace pe
