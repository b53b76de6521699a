// Launch interfaces of the attention of several query rows (trees of drafted tokens, page weights) and of accepted paths, and how
// the attention's work is cut up.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pe_check.h"
#include "pe_place.h"

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
  float* partials;  // [KV head][sequence][splits][drafts * G][D + 2] fp32 (unused when splits == 1)
  float scale;
  int num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks;
  int tile_rows, splits;
  bool is_bf16, shared;
  uint32_t* shares = nullptr;  // [num_seqs][2] where the splits are shared out by the sequences' lengths: a sequence's first one and their number
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

// Query rows that a workgroup of the attention takes: 16 or 32 of paged_rows.hip, or kWideRows of tree_wide.hip (bfloat16).  Few rows a
// workgroup make many of them, which fill the chip without splits (whose merge costs), and read K and V again and again (out of the
// second-level cache).  Measured on an MI355X, each form with as many splits as leave no compute unit two workgroups, 16 | 32 | 256, us
// (bfloat16, eight KV heads of D = 128, 4096 tokens a sequence):
//   one sequence, 32 query rows a KV head 12.9 | 15.5 | 17.3, 64 rows 14.5 | 16.2 | 18.5, 128 rows 18.9 | 18.1 | 21.4, 256 rows 27.9 | 23.1 | 28.5;
//   eight sequences, 32 rows 30.9 | 29.6 | 37.5, 64 rows 45.6 | 36.5 | 41.6, 96 rows 86.5 | 49.9 | 45.4, 128 rows 86.4 | 52.2 | 48.4, 192 rows
//   129.8 | 92.8 | 64.0; 32 sequences of 1024 to 2048 tokens, 32 rows 55.9 | 43.1 | 60.0, 64 rows 94.8 | 63.5 | 61.8, 128 rows 165.5 | 106.6 | 71.8.
constexpr int kWideRows = 256, kWideTile = 64;  // and tokens of a step
inline int tree_tile_rows(bool is_bf16, int64_t kv_rows, int rows, int compute_units) {
  const int64_t of16 = kv_rows * ((rows + 15) / 16), of32 = kv_rows * ((rows + 31) / 32);
  if (rows <= 16 || of16 * 8 <= compute_units) return 16;
  return !is_bf16 || rows <= 64 || of32 * 4 <= compute_units ? 32 : kWideRows;
}

// Splits of a row: as many as leave no compute unit two workgroups, of 128 tokens or more (of the table's, which the host knows).  More than half
// as many workgroups as compute units, or a few more than there are, leave many of these idle in the end; long rows are cut in two or three then,
// where the compute units' turns (of whole workgroups, each a part of a row) become three quarters or less.  (One / that many, us, bfloat16,
// D = 128, one query with weights: rows of 4096 tokens, 136 of them 60.3 / 54.4, 160 64.0 / 61.9, 288 135 / 115, 320 137 / 122, 384 151 / 139;
// the same down to half the length, 8192: 110 / 85.8, 114 / 96.9, 203 / 174, 212 / 183, 234 / 215.  Not with rows of 1024: 136 of them
// 18.5 / 21.9.  192 rows, which only four parts would even out: 69.8 / 72.8.  Rows of 700 tokens in such tables, eight drafts: 136 of them
// 20.3 / 23.3, 288 35.2 / 39.2.  136, 288 and 384 rows of 4096 tokens, and of half to full 8192: eight drafts x 4 heads 65.1 / 58.6, 140 / 123,
// 157 / 151, and 113 / 91.7, 206 / 182, 235 / 227; D = 64, weights, 33.1 / 31.8, 75.5 / 67.7, 84.2 / 81.5, and 64.5 / 53.4, 115 / 100, 133 / 126;
// fp32, weights, 110 / 104, 263 / 216, 285 / 261, and 213 / 156, 394 / 325, 446 / 404; fp32, D = 64, eight drafts x 4 heads 93.3 / 66.7,
// 163 / 132, 168 / 158, and 172 / 102, 249 / 196, 270 / 236.  Not the form with 256 query rows, whose records are many; 160 rows, 64 drafts x 4
// heads, one / two / three: 1024 tokens, half to full 55.2 / 74.0 / 68.0, 2048 94.1 / 124 / 108, 4096 167 / 202 / 168; 240 rows of 4096 216 / 234 /
// 246.  Where its rows are long and of unequal length three would help: 4096, half to full, 160 rows 156 / 168 / 140, 136 rows 156 / 156 / 126.)
constexpr int kLongTokens = 4096;
inline int tree_splits(bool is_bf16, int64_t kv_rows, int rows, int64_t tokens, int compute_units) {
  const int tile = tree_tile_rows(is_bf16, kv_rows, rows, compute_units);
  const int64_t groups = kv_rows * ((rows + tile - 1) / tile);
  int64_t splits = compute_units / groups;
  if (splits > tokens / 128) splits = tokens / 128;
  if (splits > 1) return splits > 64 ? 64 : (int)splits;
  const auto turns = [&](int64_t parts) { return (groups * parts + compute_units - 1) / compute_units; };
  int64_t best = 1;
  if (tile != kWideRows && tokens >= kLongTokens)
    for (int64_t parts = 2; parts <= 3; ++parts)
      if (turns(parts) * 4 <= turns(1) * parts * 3 && turns(parts) * best < turns(best) * parts) best = parts;
  return (int)best;
}

// Whether the attention and the merge of its splits are launches that the runtime takes (threads of paged_rows.hip, and of tree_wide.hip's two
// waves for every 64 rows; the merge has a workgroup for four query rows, that of page weights one for a row).
constexpr int kRowsThreads = 256, kPathThreads = 512, kMergeRows = 4;
inline bool rows_launches(const pe_cache_desc* d, int tile_rows, int rows, int splits, bool weights) {
  PlaceGrid grid;
  if (!place_grid(d->num_seqs, d->num_kv_heads, splits * ((rows + tile_rows - 1) / tile_rows), true, &grid)) return false;
  const int64_t kv_rows = (int64_t)d->num_seqs * d->num_kv_heads, merges = weights ? kv_rows : kv_rows * ((rows + kMergeRows - 1) / kMergeRows);
  return host::one_launch(grid.x, tile_rows == kWideRows ? kWideRows * 2 : kRowsThreads) && (splits == 1 || host::one_launch(merges, kRowsThreads));
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
inline size_t tree_partials_bytes(const pe_cache_desc* d, int drafts, int splits) {
  return splits > 1 ? (size_t)d->num_seqs * d->num_q_heads * drafts * splits * (d->head_dim + 2) * sizeof(float) : 0;
}
// Up to 64 sequences of tree_wide.hip have their splits shared out among them (a lane looks at a sequence; pe_rows_device.h).
inline bool tree_shares_splits(const pe_cache_desc* d, int drafts, int splits) {
  return d->num_seqs > 1 && d->num_seqs <= 64 && splits > 1 &&
         tree_tile_rows(d->dtype == PE_BF16, (int64_t)d->num_seqs * d->num_kv_heads, drafts * (d->num_q_heads / d->num_kv_heads),
                        host::compute_units()) == kWideRows;
}
inline size_t tree_workspace_bytes(const pe_cache_desc* d, int64_t drafts) {
  if (drafts < 1 || drafts > kMostDrafts) return 0;
  const int splits = tree_splits_of(d, (int)drafts);
  return tree_partials_bytes(d, (int)drafts, splits) + (tree_shares_splits(d, (int)drafts, splits) ? (size_t)d->num_seqs * 2 * sizeof(uint32_t) : 0);
}

}  // namespace pe
