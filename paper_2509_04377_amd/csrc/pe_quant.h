// Launch interfaces of the cache in 8 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pe.h"
#include "pe_check.h"
#include "pe_launch.h"

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
// Splits of a row: as many as leave no compute unit two workgroups, none shorter than 256 tokens of the table row.
inline int quant_splits(const pe_cache_desc* d) {
  if (d->decode_splits > 0) return d->decode_splits;
  const int64_t rows = (int64_t)d->num_seqs * d->num_kv_heads, tokens = (int64_t)d->max_blocks * d->block_size;
  int64_t splits = host::compute_units() / rows;
  if (splits > tokens / 256) splits = tokens / 256;
  return splits < 1 ? 1 : splits > 64 ? 64 : (int)splits;
}
inline size_t quant_workspace_bytes(const pe_cache_desc* d) {
  return decode_partials_bytes(d->num_seqs, d->num_q_heads, d->head_dim, quant_splits(d));
}

hipError_t launch_quant_decode(const QuantDecodeArgs& a, hipStream_t stream);

}  // namespace pe
