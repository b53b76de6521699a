// C-ABI layer of libpe, pages selected by a query (see include/pe.h): argument validation on the host, then kernel launches on the
// caller's stream.
#include "../../include/pe.h"

#include "pe_check.h"
#include "pe_select.h"

using namespace pe::host;

extern "C" {

int pe_page_bounds(const pe_cache_desc* desc, const void* k_pool, const int32_t* block_table, const int32_t* seq_lens,
                   int32_t recent, void* bounds_inout, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (!k_pool || !block_table || !seq_lens || !bounds_inout || recent < 0) return PE_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(bounds_inout, 16)) return PE_ERR_INVALID_ARG;
  const int64_t chunks = (int64_t)desc->head_dim * (desc->dtype == PE_F32 ? 4 : 2) / 16 * (desc->layout == PE_LAYOUT_SHARED ? desc->num_kv_heads : 1);
  if (chunks > 0x7fffffffLL || !one_launch(pe::bounds_groups(pe::bounds_per_row(recent, desc->max_blocks), (int)chunks), pe::kBoundsThreads))
    return PE_ERR_UNSUPPORTED;
  pe::BoundsArgs a;
  a.k_pool = k_pool;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.bounds = bounds_inout;
  a.recent = recent;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  return pe::launch_page_bounds(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_select_pages(const pe_cache_desc* desc, const void* q, const void* bounds, const int32_t* block_table,
                    const int32_t* seq_lens, int32_t num_pages, int32_t* block_table_out, int32_t* seq_lens_out,
                    int32_t* page_idx_out, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (!q || !bounds || !block_table || !seq_lens || !block_table_out || !seq_lens_out || num_pages < 1) return PE_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(bounds, 16)) return PE_ERR_INVALID_ARG;
  if (!one_launch(((int64_t)desc->max_blocks + pe::kFewestScored - 1) / pe::kFewestScored, pe::kScoreThreads)) return PE_ERR_UNSUPPORTED;
  const size_t rows = desc->layout == PE_LAYOUT_SHARED ? (size_t)desc->num_seqs : (size_t)desc->num_seqs * desc->num_kv_heads;
  const size_t in = rows * desc->max_blocks * 4, out = rows * num_pages * 4, lens = (size_t)desc->num_seqs * 4;
  // the rows of a sequence read what another one has already written
  if (overlap(block_table_out, out, block_table, in) || overlap(block_table_out, out, seq_lens, lens) ||
      overlap(seq_lens_out, lens, seq_lens, lens) || overlap(seq_lens_out, lens, block_table, in) ||
      (page_idx_out && (overlap(page_idx_out, out, block_table, in) || overlap(page_idx_out, out, seq_lens, lens))))
    return PE_ERR_INVALID_ARG;
  const int ws = check_workspace(workspace, workspace_bytes, pe::select_workspace_bytes(desc));
  if (ws != PE_OK) return ws;
  pe::SelectArgs a;
  a.q = q;
  a.bounds = bounds;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.table_out = block_table_out;
  a.lens_out = seq_lens_out;
  a.idx_out = page_idx_out;
  a.scores = static_cast<float*>(workspace);
  a.pages = num_pages;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.num_q_heads = desc->num_q_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  return pe::launch_select_pages(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

}  // extern "C"
