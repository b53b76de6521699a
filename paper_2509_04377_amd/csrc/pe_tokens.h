// Launch interfaces of what new tokens need before the cache: their plan (tables, slots, positions) and their rotation.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pe.h"

namespace pe {

struct PlanArgs {
  const int32_t* seq_lens;
  const int32_t* new_lens;
  const int32_t* first_positions;  // may be null
  const int32_t* free_pages;
  const int32_t* free_used;
  int32_t* block_table;
  int32_t* spare;  // may be null
  int32_t* seq_lens_out;
  int32_t* free_used_out;
  int32_t* cu_out;         // may be null
  int32_t* positions_out;  // may be null
  int64_t* slots_out;      // may be null
  int32_t* admitted;       // may be null
  int32_t* spare_used;     // may be null
  int32_t* freed_phys;     // may be null
  const int32_t* only;     // may be null
  int64_t total_tokens;
  int num_free, n_spare, budget, num_seqs, rows_per_seq, block_size, max_blocks, copies;
};
constexpr int kPlanThreads = 256;
hipError_t launch_plan_tokens(const PlanArgs& a, int compute_units, hipStream_t stream);

struct RotateArgs {
  const int32_t* positions;
  const void *q, *k, *v;
  void *q_out, *k_out;
  const int64_t* slots;  // may be null
  void *k_pool, *v_pool;
  int64_t tokens, q_stride, k_stride, v_stride, q_out_stride, k_out_stride;  // in elements
  int64_t pool_tokens;                                                       // slots of a pool
  int num_q_heads, num_kv_heads, head_dim;  // (of what there is: no queries, 0)
  bool is_bf16, shared, transpose;
};
constexpr int kRotateThreads = 256;
hipError_t launch_rotate(const RotateArgs& a, const pe_rope& rope, hipStream_t stream);

}  // namespace pe
