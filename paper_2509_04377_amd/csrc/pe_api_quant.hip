// C-ABI layer of libpe, the cache in 8 bits (see include/pe.h): argument validation on the host, then kernel launches on the caller's stream.
#include "../../include/pe.h"

#include "pe_check.h"
#include "pe_launch.h"
#include "pe_quant.h"

using namespace pe::host;

namespace {

// The five tensors of a cache.
struct Parts {
  struct { const void* p; size_t bytes; } of[5];
  bool meet(const void* p, size_t bytes) const {
    for (const auto& x : of)
      if (overlap(x.p, x.bytes, p, bytes)) return true;
    return false;
  }
};

int check_cache(const pe_cache_desc* d, const pe_quant_cache* c, Parts* parts) {
  if (c == nullptr || !c->k || !c->v || !c->scales || !c->k_tail || !c->v_tail) return PE_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 8) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16))
    return PE_ERR_INVALID_ARG;
  const size_t rows = (size_t)d->num_phys_blocks * (d->layout == PE_LAYOUT_SHARED ? (size_t)d->num_kv_heads : 1);
  const size_t pool = rows * d->block_size * d->head_dim;
  const size_t tail = (size_t)d->num_seqs * d->num_kv_heads * d->block_size * d->head_dim * (d->dtype == PE_F32 ? 4 : 2);
  *parts = Parts{{{c->k, pool}, {c->v, pool}, {c->scales, rows * 8}, {c->k_tail, tail}, {c->v_tail, tail}}};
  for (int i = 1; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(parts->of[i].p, parts->of[i].bytes, parts->of[j].p, parts->of[j].bytes)) return PE_ERR_INVALID_ARG;
  return PE_OK;
}

}  // namespace

extern "C" {

int pe_quant_pages(const pe_cache_desc* desc, const pe_quant_cache* cache, const void* k_pool, const void* v_pool,
                   const int32_t* src_table, const int32_t* seq_lens, const int32_t* block_table, float* scores_out, void* stream) {
  return pe_quant_pages_admitted(desc, cache, nullptr, k_pool, v_pool, src_table, seq_lens, block_table, scores_out, stream);
}

int pe_quant_pages_admitted(const pe_cache_desc* desc, const pe_quant_cache* cache, const int32_t* admitted, const void* k_pool,
                            const void* v_pool, const int32_t* src_table, const int32_t* seq_lens, const int32_t* block_table,
                            float* scores_out, void* stream) {
  Parts parts;
  int st = check_desc(desc);
  if (st == PE_OK) st = check_cache(desc, cache, &parts);
  if (st != PE_OK) return st;
  if (!k_pool || !v_pool || !src_table || !seq_lens || !block_table) return PE_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(scores_out, 4)) return PE_ERR_INVALID_ARG;
  const size_t page = (size_t)desc->block_size * desc->head_dim * (desc->dtype == PE_F32 ? 4 : 2);  // (how many there are is not known)
  if (parts.meet(k_pool, page) || parts.meet(v_pool, page)) return PE_ERR_INVALID_ARG;
  const size_t scored = (size_t)desc->num_seqs * desc->num_kv_heads * desc->max_blocks * 4;
  if (admitted != nullptr && (parts.meet(admitted, (size_t)desc->num_seqs * 4) ||
                              (scores_out != nullptr && overlap(admitted, (size_t)desc->num_seqs * 4, scores_out, scored))))
    return PE_ERR_INVALID_ARG;
  if (desc->num_kv_heads > 65536 || !pe::quant_pages_launches(desc)) return PE_ERR_UNSUPPORTED;
  pe::QuantPagesArgs a;
  a.cache = *cache;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.src_table = src_table;
  a.seq_lens = seq_lens;
  a.block_table = block_table;
  a.admitted = admitted;
  a.scores = scores_out;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  return pe::launch_quant_pages(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_quant_append(const pe_cache_desc* desc, const pe_quant_cache* cache, const pe_rope* rope, const int32_t* positions, const void* q,
                    void* q_out, const void* new_k, const void* new_v, int32_t* block_table, const int32_t* seq_lens,
                    int32_t* seq_lens_out, int32_t* freed_phys, const int32_t* spare, int32_t* spare_used, int32_t n_spare,
                    float* scores, void* stream) {
  Parts parts;
  int st = check_desc(desc);
  if (st == PE_OK) st = check_cache(desc, cache, &parts);
  if (st != PE_OK) return st;
  if (!new_k || !new_v || !block_table || !seq_lens || !seq_lens_out || !freed_phys || !spare || !spare_used || n_spare < 1)
    return PE_ERR_INVALID_ARG;
  if (!aligned(new_k, 16) || !aligned(new_v, 16) || !aligned(scores, 4)) return PE_ERR_INVALID_ARG;
  const size_t lens = (size_t)desc->num_seqs * 4, bytes = desc->dtype == PE_F32 ? 4 : 2;
  if (overlap(seq_lens, lens, seq_lens_out, lens)) return PE_ERR_INVALID_ARG;
  const size_t kv = (size_t)desc->num_seqs * desc->num_kv_heads * desc->head_dim * bytes;
  if (parts.meet(new_k, kv) || parts.meet(new_v, kv)) return PE_ERR_INVALID_ARG;
  if (rope != nullptr) {
    if (!rope_ok(rope, desc->head_dim) || !positions || !q || !q_out || !aligned(q, 16) || !aligned(q_out, 16)) return PE_ERR_INVALID_ARG;
    const size_t o = (size_t)desc->num_seqs * desc->num_q_heads * desc->head_dim * bytes;
    if ((q != q_out && overlap(q, o, q_out, o)) || overlap(q_out, o, new_k, kv) || overlap(q_out, o, new_v, kv) || parts.meet(q_out, o) ||
        overlap(q_out, o, positions, lens))
      return PE_ERR_INVALID_ARG;
  }
  if (desc->num_kv_heads > 65536 || (int64_t)desc->num_seqs * desc->num_kv_heads >= 1 << 23) return PE_ERR_UNSUPPORTED;
  pe::QuantAppendArgs a;
  a.cache = *cache;
  a.positions = positions;
  a.q = q;
  a.q_out = q_out;
  a.new_k = new_k;
  a.new_v = new_v;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.seq_lens_out = seq_lens_out;
  a.freed_phys = freed_phys;
  a.spare = spare;
  a.spare_used = spare_used;
  a.scores = scores;
  a.n_spare = n_spare;
  a.num_seqs = desc->num_seqs;
  a.num_kv_heads = desc->num_kv_heads;
  a.num_q_heads = desc->num_q_heads;
  a.head_dim = desc->head_dim;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  return pe::launch_quant_append(a, rope, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_quant_decode(const pe_cache_desc* desc, const pe_quant_cache* cache, const void* q, const int32_t* block_table,
                    const int32_t* seq_lens, float softmax_scale, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  Parts parts;
  int st = check_desc(desc);
  if (st == PE_OK) st = check_cache(desc, cache, &parts);
  if (st != PE_OK) return st;
  if (!q || !block_table || !seq_lens || !out) return PE_ERR_INVALID_ARG;
  const bool bf16 = desc->dtype == PE_BF16;
  if (!aligned(q, 16) || !aligned(out, bf16 ? 2 : 4) || !finite(softmax_scale)) return PE_ERR_INVALID_ARG;
  const size_t o = (size_t)desc->num_seqs * desc->num_q_heads * desc->head_dim * (bf16 ? 2 : 4);
  if ((out != q && overlap(out, o, q, o)) || parts.meet(out, o)) return PE_ERR_INVALID_ARG;
  const int splits = pe::quant_splits(desc);
  if (desc->num_kv_heads > 65536 || !pe::quant_launches(desc, splits)) return PE_ERR_UNSUPPORTED;
  const int ws = check_workspace(workspace, workspace_bytes, pe::decode_partials_bytes(desc->num_seqs, desc->num_q_heads, desc->head_dim, splits));
  if (ws != PE_OK) return ws;
  pe::QuantDecodeArgs a;
  a.cache = *cache;
  a.q = q;
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
  a.splits = splits;
  a.is_bf16 = bf16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  const int64_t groups = (int64_t)desc->num_seqs * desc->num_kv_heads * splits;
  a.waves = pe::quant_waves(desc, splits);
  a.depth = pe::quant_depth(desc, splits, a.waves);
  // the splits are merged by the last of a row to arrive where that pays (pe_decode_common.h), and where the output can hold tags before it is written
  const int heads = desc->num_q_heads / desc->num_kv_heads;
  if (splits > 1 && splits <= pe::most_arrivals(heads) && (heads > 4 ? 8 : 4) * desc->head_dim <= 128 * a.waves && groups <= 2LL * compute_units() &&
      aligned(out, 8) && out != q) {
    a.tagged = true;
    a.tag = launch_tag();
  }
  return pe::launch_quant_decode(a, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

}  // extern "C"
