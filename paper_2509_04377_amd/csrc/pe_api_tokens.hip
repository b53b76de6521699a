// C-ABI layer of libpe, the plan of new tokens and their rotation (see include/pe.h): argument validation on the host, then kernel launches on
// the caller's stream.
#include "../../include/pe.h"

#include <float.h>
#include <math.h>

#include "pe_check.h"
#include "pe_tokens.h"

using namespace pe::host;

namespace {

// The memory that `tokens` rows of `width` elements, `stride` elements apart, lie in.
size_t span(int64_t tokens, int64_t stride, int64_t width, size_t bytes) { return (size_t)((tokens - 1) * stride + width) * bytes; }

}  // namespace

extern "C" {

int pe_plan_tokens(const pe_cache_desc* desc, const int32_t* seq_lens, const int32_t* new_lens, const int32_t* first_positions,
                   int64_t total_tokens, int32_t budget_tokens, const int32_t* free_pages, int32_t num_free, const int32_t* free_used,
                   int32_t* block_table, int32_t* spare, int32_t n_spare, int32_t* seq_lens_out, int32_t* free_used_out,
                   int32_t* cu_seqlens_out, int32_t* positions_out, int64_t* slots_out, void* stream) {
  return pe_plan_tokens_ex(desc, nullptr, seq_lens, new_lens, first_positions, total_tokens, budget_tokens, free_pages, num_free, free_used,
                           block_table, spare, n_spare, seq_lens_out, free_used_out, cu_seqlens_out, positions_out, slots_out, stream);
}

int pe_plan_tokens_ex(const pe_cache_desc* desc, const pe_plan_opts* opts, const int32_t* seq_lens, const int32_t* new_lens,
                      const int32_t* first_positions, int64_t total_tokens, int32_t budget_tokens, const int32_t* free_pages, int32_t num_free,
                      const int32_t* free_used, int32_t* block_table, int32_t* spare, int32_t n_spare, int32_t* seq_lens_out,
                      int32_t* free_used_out, int32_t* cu_seqlens_out, int32_t* positions_out, int64_t* slots_out, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (!seq_lens || !new_lens || !free_pages || !free_used || !block_table || !seq_lens_out || !free_used_out) return PE_ERR_INVALID_ARG;
  if (total_tokens < 0 || total_tokens > 0x7fffffffLL || budget_tokens < 0 || num_free < 1 || n_spare < 0 || (n_spare > 0) != (spare != nullptr))
    return PE_ERR_INVALID_ARG;
  if (budget_tokens % desc->block_size != 0) return PE_ERR_INVALID_ARG;
  if (!aligned(slots_out, 8)) return PE_ERR_INVALID_ARG;
  const pe_plan_opts o = opts != nullptr ? *opts : pe_plan_opts{};
  if (o.copies < 0) return PE_ERR_INVALID_ARG;
  const bool shared = desc->layout == PE_LAYOUT_SHARED;
  const size_t S = (size_t)desc->num_seqs, per_seq = shared ? 1 : (size_t)desc->num_kv_heads;
  if (desc->num_kv_heads > 65536 || (int64_t)per_seq * ((int64_t)desc->max_blocks + n_spare) > 0x7fffffffLL) return PE_ERR_UNSUPPORTED;
  const struct { const void* p; size_t bytes; } in[] = {{seq_lens, S * 4}, {new_lens, S * 4}, {first_positions, S * 4},
                                                        {free_pages, (size_t)num_free * 4}, {free_used, 4}, {o.only, S * 4}},
      out[] = {{block_table, S * per_seq * desc->max_blocks * 4}, {spare, S * per_seq * n_spare * 4}, {seq_lens_out, S * 4}, {free_used_out, 4},
               {cu_seqlens_out, (S + 1) * 4}, {positions_out, (size_t)total_tokens * 4}, {slots_out, (size_t)total_tokens * per_seq * 8}, {o.admitted, S * 4},
               {o.spare_used, S * per_seq * 4}, {o.freed_phys, S * per_seq * 4}};
  for (size_t i = 0; i < sizeof(out) / sizeof(out[0]); ++i) {
    if (out[i].p == nullptr || out[i].bytes == 0) continue;
    for (const auto& x : in)
      if (x.p != nullptr && overlap(out[i].p, out[i].bytes, x.p, x.bytes)) return PE_ERR_INVALID_ARG;
    for (size_t j = 0; j < i; ++j)
      if (out[j].p != nullptr && overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return PE_ERR_INVALID_ARG;
  }
  pe::PlanArgs a;
  a.seq_lens = seq_lens;
  a.new_lens = new_lens;
  a.first_positions = first_positions;
  a.free_pages = free_pages;
  a.free_used = free_used;
  a.block_table = block_table;
  a.spare = spare;
  a.seq_lens_out = seq_lens_out;
  a.free_used_out = free_used_out;
  a.cu_out = cu_seqlens_out;
  a.positions_out = positions_out;
  a.slots_out = slots_out;
  a.admitted = o.admitted;
  a.spare_used = n_spare > 0 ? o.spare_used : nullptr;
  a.freed_phys = o.freed_phys;
  a.only = o.only;
  a.copies = o.copies > 1 ? o.copies : 1;
  a.total_tokens = total_tokens;
  a.num_free = num_free;
  a.n_spare = n_spare;
  a.budget = budget_tokens;
  a.num_seqs = desc->num_seqs;
  a.rows_per_seq = (int)per_seq;
  a.block_size = desc->block_size;
  a.max_blocks = desc->max_blocks;
  return pe::launch_plan_tokens(a, compute_units(), static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

int pe_rope_init(pe_rope* rope, int32_t rotary_dim, int32_t pairs, double base, int32_t scaling, double factor, double low,
                 double high, double original, double magnitude) {
  if (rope == nullptr) return PE_ERR_INVALID_ARG;
  *rope = pe_rope{};
  if (rotary_dim < 2 || rotary_dim % 2 != 0) return PE_ERR_INVALID_ARG;
  if (rotary_dim > 128) return PE_ERR_UNSUPPORTED;
  if (pairs != PE_ROPE_HALF && pairs != PE_ROPE_INTERLEAVED) return PE_ERR_INVALID_ARG;
  if (scaling != PE_ROPE_PLAIN && scaling != PE_ROPE_LINEAR && scaling != PE_ROPE_BY_PARTS) return PE_ERR_INVALID_ARG;
  if (!(base > 1.0) || !isfinite(base) || !(magnitude > 0.0) || !isfinite((float)magnitude) || !((float)magnitude > 0.f)) return PE_ERR_INVALID_ARG;
  if (scaling != PE_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return PE_ERR_INVALID_ARG;
  if (scaling == PE_ROPE_BY_PARTS && (!(low >= 0.0) || !(high > low) || !isfinite(high) || !(original > 0.0) || !isfinite(original)))
    return PE_ERR_INVALID_ARG;
  // With 64 bits of mantissa: a power, a quotient and the exponent's rounding, half a step each and the last one ln f times, leave f / 2 pi <= 0.16
  // off by less than a unit, and its rounding by half a one.
#if !defined(__HIP_DEVICE_COMPILE__)
  static_assert(LDBL_MANT_DIG >= 64, "an x86 host's long double");
#endif
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    long double f = powl((long double)base, -2.0L * i / rotary_dim);
    if (scaling == PE_ROPE_LINEAR) {
      f /= factor;
    } else if (scaling == PE_ROPE_BY_PARTS) {
      const long double g = (original * f / two_pi - low) / ((long double)high - low);
      const long double keep = g < 0.0L ? 0.0L : g > 1.0L ? 1.0L : g;
      f *= keep + (1.0L - keep) / factor;
    }
    rope->turns[i] = (uint64_t)rintl(f / two_pi * 18446744073709551616.0L);  // f <= 1: less than a sixth of a turn
  }
  rope->rotary_dim = rotary_dim;
  rope->pairs = pairs;
  rope->magnitude = (float)magnitude;
  rope->filled = 1;
  return PE_OK;
}

int pe_rotate(const pe_cache_desc* desc, const pe_rope* rope, int32_t transpose, int64_t num_tokens, const int32_t* positions,
              const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
              int64_t q_out_stride, void* k_out, int64_t k_out_stride, const int64_t* slots, void* k_pool, void* v_pool, void* stream) {
  const int st = check_desc(desc);
  if (st != PE_OK) return st;
  if (!rope_ok(rope, desc->head_dim) || num_tokens < 0) return PE_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr && (k_out != nullptr || slots != nullptr)) || (k != nullptr && !k_out && !slots))
    return PE_ERR_INVALID_ARG;
  if (num_tokens == 0) return PE_OK;
  if (positions == nullptr || (slots != nullptr && (!v || !k_pool || !v_pool))) return PE_ERR_INVALID_ARG;
  if (desc->num_q_heads > 65536 || desc->num_kv_heads > 65536) return PE_ERR_UNSUPPORTED;
  if (num_tokens > 0x7fffffffLL) return PE_ERR_UNSUPPORTED;
  const size_t bytes = desc->dtype == PE_F32 ? 4 : 2;
  const int64_t qw = (int64_t)desc->num_q_heads * desc->head_dim, kw = (int64_t)desc->num_kv_heads * desc->head_dim;
  struct Rows { const void* p; int64_t stride, width; };
  const Rows in[] = {{q, q_stride, qw}, {k, k_stride, kw}, {slots ? v : nullptr, v_stride, kw}}, out[] = {{q_out, q_out_stride, qw}, {k_out, k_out_stride, kw}};
  for (const Rows& r : {in[0], in[1], in[2], out[0], out[1]})
    if (r.p != nullptr && (!aligned(r.p, bytes) || r.stride < r.width || r.stride > (1LL << 40) / num_tokens + r.width)) return PE_ERR_INVALID_ARG;
  if (slots != nullptr && (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(slots, 8))) return PE_ERR_INVALID_ARG;
  // What is written: in place of its own input, or nowhere near anything else.  (Parts of one row a token side by side span the same memory
  // without a common byte.)
  const auto apart = [&](const Rows& a, const Rows& b) {
    if (a.p == nullptr || b.p == nullptr) return true;
    if (!overlap(a.p, span(num_tokens, a.stride, a.width, bytes), b.p, span(num_tokens, b.stride, b.width, bytes))) return true;
    if (a.stride != b.stride) return false;
    const int64_t period = a.stride * (int64_t)bytes;
    int64_t off = ((int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % period + period) % period;
    return off >= a.width * (int64_t)bytes && off + b.width * (int64_t)bytes <= period;
  };
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 3; ++j)
      if (!(i == j && out[i].p == in[j].p && out[i].stride == in[j].stride) && !apart(out[i], in[j])) return PE_ERR_INVALID_ARG;
  if (!apart(out[0], out[1])) return PE_ERR_INVALID_ARG;
  const size_t slot_bytes = (size_t)num_tokens * 8 * (desc->layout == PE_LAYOUT_SHARED ? 1 : desc->num_kv_heads);
  for (const Rows& r : out) {
    if (r.p == nullptr) continue;
    const size_t all = span(num_tokens, r.stride, r.width, bytes);
    if (overlap(r.p, all, positions, (size_t)num_tokens * 4) || (slots != nullptr && overlap(r.p, all, slots, slot_bytes))) return PE_ERR_INVALID_ARG;
  }
  if (slots != nullptr) {
    const size_t pool = (size_t)desc->num_phys_blocks * desc->block_size * desc->head_dim * bytes *
                        (desc->layout == PE_LAYOUT_SHARED ? desc->num_kv_heads : 1);
    if (overlap(k_pool, pool, v_pool, pool)) return PE_ERR_INVALID_ARG;
    for (const void* p : {(const void*)k_pool, (const void*)v_pool})
      for (const Rows& r : {in[0], in[1], in[2], out[0], out[1]})
        if (r.p != nullptr && overlap(p, pool, r.p, span(num_tokens, r.stride, r.width, bytes))) return PE_ERR_INVALID_ARG;
  }
  pe::RotateArgs a;
  a.positions = positions;
  a.q = q;
  a.k = k;
  a.v = slots ? v : nullptr;
  a.q_out = q_out;
  a.k_out = k_out;
  a.slots = slots;
  a.k_pool = slots ? k_pool : nullptr;
  a.v_pool = slots ? v_pool : nullptr;
  a.tokens = num_tokens;
  a.q_stride = q ? q_stride : 0;
  a.k_stride = k ? k_stride : 0;
  a.v_stride = slots ? v_stride : 0;
  a.q_out_stride = q_out ? q_out_stride : 0;
  a.k_out_stride = k_out ? k_out_stride : 0;
  a.pool_tokens = desc->num_phys_blocks * desc->block_size;
  a.num_q_heads = q ? desc->num_q_heads : 0;
  a.num_kv_heads = k ? desc->num_kv_heads : 0;
  a.head_dim = desc->head_dim;
  a.is_bf16 = desc->dtype == PE_BF16;
  a.shared = desc->layout == PE_LAYOUT_SHARED;
  a.transpose = transpose != 0;
  if (a.num_q_heads + a.num_kv_heads == 0) return PE_OK;
  return pe::launch_rotate(a, *rope, static_cast<hipStream_t>(stream)) == hipSuccess ? PE_OK : PE_ERR_HIP;
}

}  // extern "C"
