// Launch interfaces of the cache in 8 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pe.h"
#include "pe_check.h"
#include "pe_launch.h"
#include "pe_place.h"

namespace pe {

struct QuantPagesArgs {
  pe_quant_cache cache;
  const void* k_pool;
  const void* v_pool;
  const int32_t* src_table;
  const int32_t* seq_lens;
  const int32_t* block_table;
  float* scores;  // may be null
  int num_seqs, num_kv_heads, head_dim, block_size, max_blocks;
  bool is_bf16, shared;
  const int32_t* admitted;  // may be null
};
// false: a launch that the runtime does not take
bool quant_pages_launches(const pe_cache_desc* d);
hipError_t launch_quant_pages(const QuantPagesArgs& a, hipStream_t stream);

struct QuantAppendArgs {
  pe_quant_cache cache;
  const int32_t* positions;  // with `rope`
  const void* q;
  void* q_out;
  const void* new_k;
  const void* new_v;
  int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* seq_lens_out;
  int32_t* freed_phys;
  const int32_t* spare;
  int32_t* spare_used;
  float* scores;  // may be null
  int n_spare, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks;
  bool is_bf16, shared;
};
hipError_t launch_quant_append(const QuantAppendArgs& a, const pe_rope* rope, hipStream_t stream);

struct QuantDecodeArgs {
  pe_quant_cache cache;
  const void* q;
  const int32_t* block_table;
  const int32_t* seq_lens;
  void* out;
  float* partials;
  float scale;
  int num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, max_blocks;
  int splits, waves, depth;
  bool is_bf16, shared;
  bool tagged = false;  // splits merged by the last of a row to arrive
  uint64_t tag = 0;
};
// Splits of a row.  The host sees the length of a table row, not of the sequences, so a count has to pay on full rows and on rows of unequal
// length (37 tokens to all; four query heads a KV head, us, best count / others; measured on an MI355X, fp32 the same order):
//   - up to half as many rows as compute units: as many as leave no compute unit two workgroups, of 128 tokens or more (64 rows of D = 128 x
//     1024 in four 6.7, x 4096 in four 12.5; eight rows x 4096 in 32 6.7, in sixteen 7.1), but not a few more than those that need no merge launch
//     (two rows of D = 64 x 1649 in thirteen 5.8, in twelve 5.3), two only of 512 or more (128 rows x 1024 in two 8.5, x 512
//     whole 6.4 / 6.8); rows of 32 KiB of K whole (eight of D = 64 x 512 whole 4.7 / 4.8, of D = 128 x 512 in four 5.3 / 5.9 whole);
//   - more, of 2048 tokens or more: three up to five eighths of the compute units (D = 128, 160 rows x 2048 in three 15.3, whole 16.1, ragged 11.6 / 13),
//     four up to three quarters (192 rows x 2048 full in four 18.1, whole 17.1, ragged 12.7 / 15), else whole (224 rows 18.9, in three 20.9, ragged
//     15.4 / 14.3); shorter ones whole (160 rows x 1024 9.8, in three 10.2, ragged 8.8 / 8.7);
//   - a few more rows than compute units, of 2048 or more, four (264 rows of D = 64 x 2048 14.4, whole 16.7; of D = 128 x 4096 48.4 / 58; not 384 rows
//     x 2048 of D = 64: whole 17.4, in two 18.4).
inline int quant_splits(const pe_cache_desc* d) {
  if (d->decode_splits > 0) return d->decode_splits;
  const int64_t rows = (int64_t)d->num_seqs * d->num_kv_heads, tokens = (int64_t)d->max_blocks * d->block_size;
  const int64_t cus = host::compute_units(), fit = cus / rows;
  if (tokens * d->head_dim <= 32768) return 1;
  if (fit < 2) {
    if (tokens < 2048) return 1;
    if (rows > cus) return rows * 10 <= cus * 13 ? 4 : 1;
    return rows * 8 <= cus * 5 ? 3 : rows * 4 <= cus * 3 ? 4 : 1;
  }
  int64_t splits = tokens / (fit == 2 ? 512 : 128);
  if (splits > fit) splits = fit;
  const int most = most_arrivals(d->num_q_heads / d->num_kv_heads);
  if (splits > most && splits <= most + 4) splits = most;
  return splits < 1 ? 1 : splits > 64 ? 64 : (int)splits;
}

// The workgroup: eight waves, four where split rows make more workgroups than compute units (192 rows of D = 128 x 2048, ragged, in four 12.7, with eight
// waves 14.6), and tiles in flight a wave: one (256 rows of D = 128 x 2048 21.4, two 21.5; 64 x 1024 in four 6.75 / 6.9), two for D = 64 in long
// pieces, whose wave-loads are half as long (256 rows x 2048 12.3, one 13.6; 64 rows x 4096 in four 9.0 / 9.4; pieces of 256 5.5, two 6.3).  The
// order is the same where the pages come from memory and not from the caches that a repeated step finds full (256 rows x 2048: D = 128 24.8, two
// 25.5; D = 64 14.7, one 15.3).
inline int quant_waves(const pe_cache_desc* d, int splits) {
  return splits > 1 && (int64_t)d->num_seqs * d->num_kv_heads * splits > host::compute_units() ? 4 : 8;
}
inline int quant_depth(const pe_cache_desc* d, int splits, int waves) {
  return d->head_dim == 64 && waves == 8 && (int64_t)d->max_blocks * d->block_size / splits >= 1024 ? 2 : 1;
}

// Whether the attention and the merge of its splits (a workgroup of up to eight waves for a query row) are launches that the runtime takes.
inline bool quant_launches(const pe_cache_desc* d, int splits) {
  PlaceGrid grid;
  if (!place_grid(d->num_seqs, d->num_kv_heads, splits, true, &grid)) return false;
  return host::one_launch(grid.x, quant_waves(d, splits) * 64) && (splits == 1 || host::one_launch((int64_t)d->num_seqs * d->num_q_heads, 512));
}

inline size_t quant_workspace_bytes(const pe_cache_desc* d) {
  return decode_partials_bytes(d->num_seqs, d->num_q_heads, d->head_dim, quant_splits(d));
}

hipError_t launch_quant_decode(const QuantDecodeArgs& a, hipStream_t stream);

}  // namespace pe
