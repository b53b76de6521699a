// C-ABI layer of libpe, trees of drafted tokens and page weights (see include/pe.h): argument validation on the host, then kernel launches on the
// caller's stream.
#include "../../include/pe.h"

#include "pe_check.h"
#include "pe_rows.h"

using namespace pe::host;

extern "C" {

int pe_tree_decode(const pe_cache_desc* desc, int32_t num_drafts, const void* q, const void* k_draft, const void* v_draft,
                   const int32_t* draft_lens, const uint64_t* tree_mask, const void* k_pool, const void* v_pool,
                   const int32_t* block_table, const int32_t* seq_lens, float softmax_scale, void* out, void* workspace,
                   size_t workspace_bytes, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (num_drafts < 1) return PE_ERR_INVALID_ARG;
  if (num_drafts > pe::kMostDrafts) return PE_ERR_UNSUPPORTED;
  if (!q || !k_draft || !v_draft || !tree_mask || !k_pool || !v_pool || !block_table || !seq_lens || !out) return PE_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(q, 16) || !aligned(k_draft, 16) || !aligned(v_draft, 16) ||
      !aligned(tree_mask, 8) || !aligned(out, desc->dtype == PE_F32 ? 4 : 2))
    return PE_ERR_INVALID_ARG;
  if (!finite(softmax_scale)) return PE_ERR_INVALID_ARG;
  if (desc->num_kv_heads > 65536) return PE_ERR_UNSUPPORTED;
  if ((int64_t)desc->num_seqs * desc->num_q_heads * num_drafts > 0x7fffffffLL / 4) return PE_ERR_UNSUPPORTED;
  const int rows = num_drafts * (desc->num_q_heads / desc->num_kv_heads), splits = pe::tree_splits_of(desc, num_drafts);
  const int tile_rows =
      pe::tree_tile_rows(desc->dtype == PE_BF16, (int64_t)desc->num_seqs * desc->num_kv_heads, rows, compute_units());
  if (!pe::rows_launches(desc, tile_rows, rows, splits, false)) return PE_ERR_UNSUPPORTED;
  const size_t head = (size_t)desc->num_seqs * num_drafts * desc->head_dim * (desc->dtype == PE_F32 ? 4 : 2);
  const size_t o = head * desc->num_q_heads, kv = head * desc->num_kv_heads;
  if ((out != q && overlap(out, o, q, o)) || overlap(out, o, k_draft, kv) || overlap(out, o, v_draft, kv)) return PE_ERR_INVALID_ARG;
  const int ws = check_workspace(workspace, workspace_bytes, pe::tree_workspace_bytes(desc, num_drafts));
  if (ws != PE_OK) return ws;
  pe::RowsArgs a;
  a.q = q;
  a.k_draft = k_draft;
  a.v_draft = v_draft;
  a.draft_lens = draft_lens;
  a.mask = tree_mask;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.out = out;
  a.partials = static_cast<float*>(workspace);
  a.scale = softmax_scale;
  a.drafts = num_drafts;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.num_q_heads = desc->num_q_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  a.tile_rows = tile_rows;
  a.splits = splits;
  if (pe::tree_shares_splits(desc, num_drafts, splits))
    a.shares = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + pe::tree_partials_bytes(desc, num_drafts, splits));
  return pe::launch_paged_rows(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_paged_decode_weights(const pe_cache_desc* desc, const void* q, const void* k_pool, const void* v_pool,
                            const int32_t* block_table, const int32_t* seq_lens, float softmax_scale, float decay,
                            const float* weights_in, float* weights_out, void* out, void* workspace, size_t workspace_bytes,
                            void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (!q || !k_pool || !v_pool || !block_table || !seq_lens || !weights_out || !out) return PE_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(q, 16) || !aligned(out, desc->dtype == PE_F32 ? 4 : 2) ||
      !aligned(weights_in, 4) || !aligned(weights_out, 4))
    return PE_ERR_INVALID_ARG;
  if (!finite(softmax_scale) || !(decay >= 0.f && decay <= 1.f)) return PE_ERR_INVALID_ARG;
  const int splits = pe::weights_splits_of(desc);
  if (desc->num_kv_heads > 65536 || splits == 0 || !pe::rows_launches(desc, 16, desc->num_q_heads / desc->num_kv_heads, splits, true))
    return PE_ERR_UNSUPPORTED;
  const size_t o = (size_t)desc->num_seqs * desc->num_q_heads * desc->head_dim * (desc->dtype == PE_F32 ? 4 : 2);
  const size_t w = (size_t)desc->num_seqs * desc->num_kv_heads * desc->max_blocks * 4;
  if ((out != q && overlap(out, o, q, o)) || overlap(weights_out, w, out, o) || overlap(weights_out, w, q, o)) return PE_ERR_INVALID_ARG;
  if (weights_in && ((weights_in != weights_out && overlap(weights_out, w, weights_in, w)) || overlap(weights_in, w, out, o)))
    return PE_ERR_INVALID_ARG;
  const int ws = check_workspace(workspace, workspace_bytes, pe::weights_workspace_bytes(desc));
  if (ws != PE_OK) return ws;
  pe::RowsArgs a;
  a.q = q;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.out = out;
  a.partials = static_cast<float*>(workspace);
  a.scale = softmax_scale;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.num_q_heads = desc->num_q_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  a.tile_rows = 16;
  a.splits = splits;
  a.weights_in = weights_in;
  a.weights_out = weights_out;
  if (splits > 1) a.page_sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + pe::weights_partials_bytes(desc, splits));
  a.decay = decay;
  a.part_bytes = pe::weights_part_bytes(desc, splits);
  return pe::launch_paged_rows(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_append_path(const pe_cache_desc* desc, int32_t num_drafts, const void* k_draft, const void* v_draft, const int32_t* path,
                   int32_t max_path, const int32_t* path_lens, int32_t* path_done, void* k_pool, void* v_pool, int32_t* block_table,
                   int32_t* seq_lens, int32_t* freed_phys, const int32_t* spare, int32_t* spare_used, int32_t n_spare, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (num_drafts < 1 || max_path < 1 || n_spare < 1) return PE_ERR_INVALID_ARG;
  if (desc->num_kv_heads > 65536 || !one_launch(desc->num_seqs, pe::kPathThreads)) return PE_ERR_UNSUPPORTED;
  if (!k_draft || !v_draft || !path || !path_lens || !path_done || !k_pool || !v_pool || !block_table || !seq_lens || !freed_phys ||
      !spare || !spare_used)
    return PE_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(k_draft, 16) || !aligned(v_draft, 16)) return PE_ERR_INVALID_ARG;
  pe::PathArgs a;
  a.k_draft = k_draft;
  a.v_draft = v_draft;
  a.path = path;
  a.path_lens = path_lens;
  a.path_done = path_done;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.freed_phys = freed_phys;
  a.spare = spare;
  a.spare_used = spare_used;
  a.drafts = num_drafts;
  a.max_path = max_path;
  a.n_spare = n_spare;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  return pe::launch_append_path(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

}  // extern "C"
