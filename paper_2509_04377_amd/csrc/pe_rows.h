// Launch interfaces of the attention of several query rows (trees of drafted tokens, page weights) and of accepted paths, and how
// the attention's work is cut up.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pe_check.h"

namespace pe {

constexpr int kMostDrafts = PE_MAX_DRAFTS;  // a draft's mask is one word

constexpr int kRoundTokens = 128;  // dealt out to a split together: no page is longer

struct RowsArgs {
  const void* q;
  const void* k_pool;
  const void* v_pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  void* out;
  float* partials;  // [rows][splits][drafts * G][D + 2] fp32 (unused when splits == 1)
  float scale;
  int num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks;
  int tile_rows, splits;
  bool is_bf16, shared;
  // trees of drafts
  int drafts = 1;
  const void* k_draft = nullptr;
  const void* v_draft = nullptr;
  const int32_t* draft_lens = nullptr;  // may be null
  const uint64_t* mask = nullptr;
  // page weights (one query a sequence)
  const float* weights_in = nullptr;  // may be null
  float* weights_out = nullptr;       // null: a tree
  float* page_sums = nullptr;         // [rows][max_blocks][G] fp32 (unused when splits == 1)
  float decay = 0.f;
  size_t part_bytes = 0;              // LDS for the parts of a split
};
hipError_t launch_paged_rows(const RowsArgs& a, hipStream_t stream);

struct PathArgs {
  const void* k_draft;
  const void* v_draft;
  const int32_t* path;
  const int32_t* path_lens;
  int32_t* path_done;
  void* k_pool;
  void* v_pool;
  int32_t* block_table;
  int32_t* seq_lens;
  int32_t* freed_phys;
  const int32_t* spare;
  int32_t* spare_used;
  int drafts, max_path, n_spare, num_seqs, num_kv_heads, head_dim, block_size, max_blocks;
  bool is_bf16, shared;
};
hipError_t launch_append_path(const PathArgs& a, hipStream_t stream);

// Query rows that a workgroup of the attention takes.
inline int tree_tile_rows(bool is_bf16, int rows) {
  return rows <= 16 ? 16 : rows <= 32 || !is_bf16 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
}

inline int tree_splits(bool is_bf16, int64_t kv_rows, int rows, int64_t tokens, int compute_units) {
  const int tile = tree_tile_rows(is_bf16, rows);
  const int64_t groups = kv_rows * ((rows + tile - 1) / tile);
  int64_t splits = (compute_units + groups - 1) / groups;
  const int64_t by_len = tokens / 256 < 1 ? 1 : tokens / 256;
  if (splits > by_len) splits = by_len;
  return splits > 64 ? 64 : (int)splits;
}

// Page weights: the parts of a split lie in LDS, 8 bytes for every 16 tokens and query head, beside what the waves' states take.
constexpr size_t kMostPartBytes = 30 << 10;
inline size_t weights_part_bytes(const pe_cache_desc* d, int splits) {
  const int64_t rounds = ((int64_t)d->max_blocks * d->block_size + kRoundTokens - 1) / kRoundTokens;
  return (size_t)((rounds + splits - 1) / splits) * (kRoundTokens / 16) * (d->num_q_heads / d->num_kv_heads) * 8;
}
// The splits of a row that a call for page weights uses; 0: the table rows are too long.
inline int weights_splits_of(const pe_cache_desc* d) {
  int splits = d->decode_splits > 0 ? d->decode_splits
                                    : tree_splits(d->dtype == PE_BF16, (int64_t)d->num_seqs * d->num_kv_heads, d->num_q_heads / d->num_kv_heads,
                                                  (int64_t)d->max_blocks * d->block_size, host::compute_units());
  const int64_t rounds = ((int64_t)d->max_blocks * d->block_size + kRoundTokens - 1) / kRoundTokens;
  const int64_t held = (int64_t)(kMostPartBytes / (kRoundTokens / 16 * 8)) / (d->num_q_heads / d->num_kv_heads);  // rounds of a split
  if ((rounds + held - 1) / held > 256) return 0;
  return splits * held < rounds ? (int)((rounds + held - 1) / held) : splits;
}
inline size_t weights_partials_bytes(const pe_cache_desc* d, int splits) {
  return splits > 1 ? ((size_t)d->num_seqs * d->num_q_heads * splits * (d->head_dim + 2) * sizeof(float) + 255) / 256 * 256 : 0;
}
inline size_t weights_workspace_bytes(const pe_cache_desc* d) {
  const int splits = weights_splits_of(d);
  return splits > 1 ? weights_partials_bytes(d, splits) + (size_t)d->num_seqs * d->num_q_heads * d->max_blocks * sizeof(float) : 0;
}

// The splits of a row that a call with `drafts` drafts uses, and the workspace that their partials take.
inline int tree_splits_of(const pe_cache_desc* d, int drafts) {
  if (d->decode_splits > 0) return d->decode_splits;
  return tree_splits(d->dtype == PE_BF16, (int64_t)d->num_seqs * d->num_kv_heads, drafts * (d->num_q_heads / d->num_kv_heads),
                     (int64_t)d->max_blocks * d->block_size, host::compute_units());
}
inline size_t tree_workspace_bytes(const pe_cache_desc* d, int64_t drafts) {
  if (drafts < 1 || drafts > kMostDrafts) return 0;
  const int splits = tree_splits_of(d, (int)drafts);
  return splits > 1 ? (size_t)d->num_seqs * d->num_q_heads * drafts * splits * (d->head_dim + 2) * sizeof(float) : 0;
}

}  // namespace pe
