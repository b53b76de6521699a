// Launch interfaces of the calls that bound pages' keys and select pages by a query.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pe_check.h"

namespace pe {

struct BoundsArgs {
  const void* k_pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  void* bounds;
  int recent;  // 0: every full page; n: the n most recently filled ones of each row
  int num_seqs, num_kv_heads, head_dim, block_size, max_blocks;
  bool is_bf16, shared;
};
hipError_t launch_page_bounds(const BoundsArgs& a, hipStream_t stream);

// Workgroups for the pages of a row: a thread has 16 bytes of every token of one page.
constexpr int kBoundsThreads = 256;
inline int64_t bounds_groups(int per_row, int chunks) { return ((int64_t)per_row * chunks + kBoundsThreads - 1) / kBoundsThreads; }
inline int bounds_per_row(int recent, int max_blocks) { return recent > 0 && recent < max_blocks ? recent : max_blocks; }

// Pages of a row that can be scored: in workgroups of eight pages (fp32, D = 128, several heads a decision) the fewest.
constexpr int kScoreThreads = 256, kFewestScored = 8;

// Scores of rows of one head a decision: sixteen loads a wave, in registers that leave four waves a SIMD, where there are two such workgroups a
// compute unit or more; eight where there are fewer, or several heads a decision.  (bf16, D = 128, the whole call with sixteen / eight: 32
// rows of 4096 pages 25.8 / 27.6 us, 256 of 1024 39.6 / 43.4, 8 of 4096 17.0 / 17.2, 8 of 1024 11.7 / 10.6; eight heads a decision, 2 rows of
// 2048 22.0 / 16.0.)
constexpr int scored_by_sixteen(int head_dim, bool is_bf16) {  // pages of a workgroup: a load is 16 bytes a lane, a page's bounds 2 D elements
  return kScoreThreads * 16 * 16 / (2 * head_dim * (is_bf16 ? 2 : 4));
}
inline bool many_scores(int64_t rows, int max_blocks, int head_dim, bool is_bf16, int compute_units) {
  const int64_t each = scored_by_sixteen(head_dim, is_bf16);
  return rows * ((max_blocks + each - 1) / each) >= 2 * compute_units;
}

struct SelectArgs {
  const void* q;
  const void* bounds;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* idx_out;  // may be null
  float* scores;     // workspace: [rows][max_blocks]
  int pages;         // selected ones of a row, at most
  int num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks;
  bool is_bf16, shared;
};
hipError_t launch_select_pages(const SelectArgs& a, hipStream_t stream);

// One score for every table entry.
inline size_t select_workspace_bytes(const pe_cache_desc* d) {
  const int64_t rows = d->layout == PE_LAYOUT_SHARED ? d->num_seqs : (int64_t)d->num_seqs * d->num_kv_heads;
  return (size_t)rows * d->max_blocks * sizeof(float);
}

}  // namespace pe
