// What the kernels for several query rows share: their arguments and small steps.
#pragma once

#include "pe_decode_common.h"
#include "pe_rows.h"

namespace pe {

constexpr float kNegInf = -__builtin_inff();
constexpr float kGrow = 3.f;  // how far above the largest logit (log2) a reference is set

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

// Two probabilities as two bfloat16 terms each: hi next to p, lo next to what hi leaves (which is exact in fp32), to nearest both, so that
// hi + lo is within 2^-17 of p and as often above as below.  (Cut off instead of rounded, in as many instructions, they were up to 2^-15 short
// and 2^-17 on average, which all of a row's tokens have in common.)
struct Terms {
  uint32_t hi, lo;
};
__device__ __forceinline__ Terms terms_of(float p0, float p1) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
  Terms t;
  t.hi = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{p0, p1}), bf16x2_t));
  const float r0 = p0 - __uint_as_float(t.hi << 16), r1 = p1 - __uint_as_float(t.hi & 0xffff0000u);
  t.lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{r0, r1}), bf16x2_t));
  return t;
}

// What a wave needs before its first load comes first (the leading arguments are in scalar registers when it starts).
struct RowsParams {
  const int32_t *seq_lens, *block_table;
  const void *k_pool, *v_pool;
  int num_kv_heads, max_blocks;  // max_blocks < 0: a table row is a sequence's
  uint32_t inv_heads;
  uint32_t shape;                // log2 of the page size, query heads per KV head, order of the workgroups, splits
  int tiles, drafts;             // workgroups for the query rows of a row; queries of a sequence
  const void* q;
  float scale_log2e;
  float decay;
  const int32_t* draft_lens;     // or null: every sequence has all of them
  const uint64_t* mask;
  const void *k_draft, *v_draft;
  void* out;
  float* partials;
  const float* weights_in;       // or null
  float* weights_out;
  float* page_sums;              // [rows][max_blocks][G], where there are several splits
  int num_seqs;
  uint32_t* shares;              // [num_seqs][2], or null: every sequence has the same number of splits
};

__device__ __forceinline__ int drafts_of(const RowsParams& p, int s) {
  if (p.draft_lens == nullptr) return p.drafts;
  const int have = p.draft_lens[s];
  return have < 0 ? 0 : have < p.drafts ? have : p.drafts;
}
__device__ __forceinline__ int length_of(const RowsParams& p, int s, int max_blocks, int log2_block) {
  const int len = p.seq_lens[s];
  const int64_t most = (int64_t)max_blocks << log2_block;  // (a longer row is a caller error: its table ends here)
  return len < 0 ? 0 : len < most ? len : (int)most;
}

// Splits by the lengths of up to 64 sequences: of the num_seqs * splits that the launch has for a KV head a sequence gets one for every t of
// its tiles of kTile tokens (the drafts are one), with the smallest t (or a few percent more, in the long run) for which they suffice.  The
// lengths are on the device, so every wave works this out for itself: a few steps, as t begins where they would suffice without remainders.
// The launch that merges the splits reads what the first of a sequence's notes.
// (64 drafts x 4 heads, eight sequences of 4001 to 8192 tokens, eight KV heads of D = 128: the longest of the 256 workgroups has 27 tiles where
// four splits a sequence give it 32, 98.8 us instead of 105.6.)
// The splits up to and including those of sequence `lane`.
__device__ __forceinline__ uint32_t splits_upto(const RowsParams& p, int max_blocks, int log2_block, int tile, int lane) {
  uint32_t units = 0u;
  if (lane < p.num_seqs && drafts_of(p, lane) > 0) units = ((uint32_t)length_of(p, lane, max_blocks, log2_block) + tile - 1) / tile + 1u;
  const uint32_t have = (uint32_t)(p.num_seqs * shape_splits(p.shape));
  const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum_u32(units), kWave - 1);
  for (uint32_t t = all > have ? (all + have - 1) / have : 1u;; t += 1u + (t >> 5)) {  // (with t the most tiles of all, one a sequence suffices)
    const uint32_t upto = wave_prefix_sum_u32((units + t - 1u) / t);
    if ((uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1) <= have) return upto;
  }
}

// The grid for `rows` query rows a workgroup, and what of the arguments goes with it.
inline bool rows_grid(const RowsArgs& a, int rows, RowsParams* p, dim3* blocks) {
  p->tiles = (a.drafts * shape_group(p->shape) + rows - 1) / rows;
  PlaceGrid grid;
  if (!place_grid(a.num_seqs, a.num_kv_heads, a.splits * p->tiles, true, &grid)) return false;
  p->shape |= (grid.xcd ? kShapeXcd : 0u) | (grid.linear ? kShapeLinear : 0u);
  p->inv_heads = grid.inv_heads;
  *blocks = dim3(grid.x, grid.y);
  return true;
}

// The attention of trees with many query rows, without the merge of the splits (tree_wide.hip).
hipError_t launch_tree_wide(const RowsArgs& a, RowsParams p, hipStream_t stream);

}  // namespace pe
