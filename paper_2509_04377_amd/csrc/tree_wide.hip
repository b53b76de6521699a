// Attention of a tree of drafted tokens over a paged bfloat16 cache, for many query rows: more than 32 share the K and V of a row.
//
// The products count here, not the traffic: 256 query rows ask for 256 operations a byte of the cache.  (64 drafts x 4 heads over eight caches of
// 4001 to 8192 tokens of D = 128, eight KV heads: 88 us and 10 for the merge, 500 TFLOP/s and half as many again for the low terms; the matrix
// units are busy for 48 % of it, as are the vector units, at the 1.7 GHz that are left of the clock.)  A workgroup owns 32 query rows a
// wave and one split of the tokens (tiles of 64, the drafts are the last one); K and V of a tile go through LDS once for all its waves,
// which read them as operands of the 32 x 32 x 16 products.  The tile behind the next one is on its way to registers while one is computed
// out of one half of LDS and the next is put into the other; one barrier a tile.
//
// With lane l = 32*h + n:
//   QK (A = K, B = Q): C[m][n] = <k_m, q_n>.  Lane l reads 16 bytes of token n (as row m), chunk 2*j + h; a token's chunks lie in LDS in an
//   order of their own (chunk ^ token), so that neighbouring tokens' do not meet in the same banks.  Lane l is left with tokens
//   8*(i/4) + 4*h + i%4 of query n, i < 16.
//   PV (A = V transposed, B = P): a product contracts 16 tokens, lane half h those that it has: registers 8*c .. 8*c + 7 of the logits.  Row m
//   of A is element 32*e + m in product e; the reads that turn 16 elements of four tokens over 16 lanes bring it out of LDS as it lies.
//
// Probabilities go into the product as two bfloat16 terms, as in paged_rows.hip, and the softmax is that one too.  (In one term, rounded, those
// drafts took 90 us where two took 104, and the outputs were sqrt(2) times as far from 64 bits: their own rounding, and as much again.)
// Measured against it and not better: tiles of 128 tokens (144 us where 64 took 123), two workgroups of four waves a compute unit (the
// same), half of the waves a phase behind the others (109 / 99), the low terms by dot products (103 / 98).
#include "pe_rows_device.h"

namespace pe {
namespace {

constexpr int kTile = kWideTile;
constexpr int WAVES = kWideRows / 32, NT = WAVES * kWave;
static_assert(NT == kWideRows * 2, "what the host counts with");

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

template <int P>
struct Parity {
  static constexpr int value = P;
};

template <int D>
__global__ __launch_bounds__(NT, 2) void tree_wide_kernel(const RowsParams p) {
  constexpr int CPT = D / 8;                 // 16-byte chunks of a token
  constexpr int NL = kTile * CPT / NT;       // 16-byte chunks of K (and of V) that a lane brings
  constexpr int CH = D / 16;                 // products of QK
  constexpr int E = D / 32;                  // elements of V that a lane reads of a token
  static_assert(NL * NT == kTile * CPT, "whole chunks");
  __shared__ uint4 sk[2][kTile * CPT], sv[2][kTile * CPT];

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int h = lane >> 5, n = lane & 31, tid = (int)threadIdx.x;
  const int log2_block = shape_log2_block(p.shape), group = shape_group(p.shape);
  int splits = shape_splits(p.shape);
  const Place at = place_at(blockIdx.x, blockIdx.y, (p.shape & kShapeXcd) != 0, (p.shape & kShapeLinear) != 0, splits * p.tiles, p.num_kv_heads,
                            p.inv_heads);
  const bool shared = p.max_blocks < 0, several = splits > 1;
  const int max_blocks = shared ? -p.max_blocks : p.max_blocks;
  const int hk = at.head;
  int s = at.seq, split = at.split / p.tiles;
  const int tile0 = at.split - split * p.tiles;
  const int64_t slot = ((int64_t)hk * p.num_seqs + s) * splits + split;  // of its record
  if (p.shares != nullptr) {
    const uint32_t mine = (uint32_t)(s * splits + split);
    const uint32_t upto = splits_upto(p, max_blocks, log2_block, kTile, lane);
    s = __builtin_amdgcn_readfirstlane((int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= mine)));
    if (s >= p.num_seqs) return;  // more than are needed
    const uint32_t first = s > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, s - 1) : 0u;
    splits = __builtin_amdgcn_readfirstlane((int)((uint32_t)__builtin_amdgcn_readlane((int)upto, s) - first));
    split = __builtin_amdgcn_readfirstlane((int)(mine - first));
    if (split == 0 && at.head == 0 && threadIdx.x == 0) *reinterpret_cast<uint2*>(p.shares + 2 * s) = make_uint2(first, (uint32_t)splits);
  }
  // (read only while the launch runs: scalar loads, which the barriers would otherwise forbid)
  const auto* table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
      reinterpret_cast<uintptr_t>(p.block_table + (shared ? (int64_t)s : (int64_t)s * p.num_kv_heads + hk) * max_blocks));
  const int drafts = drafts_of(p, s), rows = drafts * group, row0 = tile0 * kWideRows;
  if (row0 >= rows) return;
  const int len = length_of(p, s, max_blocks, log2_block);
  const int cached = len / kTile + (len % kTile != 0), tiles = cached + 1;

  // ---- staging ------------------------------------------------------------------------------------------------------------
  // A wave brings NL runs of K and of V of a tile, TPL token rows each, which lie in one page: its place is looked up with scalar loads.
  constexpr int TPL = kWave / CPT;
  const int t_lane = lane / CPT, c_of = lane % CPT;
  const uint32_t token_bytes = (uint32_t)(shared ? p.num_kv_heads : 1) * (D * 2), draft_bytes = (uint32_t)p.num_kv_heads * (D * 2);
  const uint32_t lane_off = (uint32_t)t_lane * token_bytes + (uint32_t)c_of * 16u;
  // (the drafts' places as distances from the pools': a choice between two arguments would load the chosen one every time)
  const int64_t k_far = static_cast<const char*>(p.k_draft) - static_cast<const char*>(p.k_pool);
  const int64_t v_far = static_cast<const char*>(p.v_draft) - static_cast<const char*>(p.v_pool);
  const auto run_of = [&](int i) { return (i * WAVES + wave) * TPL; };  // the first token of run i in its tile
  int ids[NL];
  const auto lookup = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int64_t j = ((int64_t)tile * kTile + run_of(i)) >> log2_block;
      ids[i] = table[j < max_blocks ? (int)j : max_blocks - 1];
    }
  };
  uint4 kr[NL], vr[NL];  // the tile behind the next one
  const auto fetch = [&](int tile) __attribute__((always_inline)) {  // (what is no token, or no tile, reads one that is)
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      int64_t base;
      uint32_t off = lane_off;
      const bool pool = tile < cached;
      if (pool) {
        const int slot = (int)(((int64_t)tile * kTile + run_of(i)) & ((1 << log2_block) - 1));
        base = (((int64_t)(ids[i] < 0 ? 0 : ids[i]) << log2_block) + slot) * token_bytes + (shared ? hk * (D * 2) : 0);
      } else {
        const int t = run_of(i) + t_lane;
        off = (uint32_t)(t < drafts ? t : 0) * draft_bytes + (uint32_t)c_of * 16u;
        base = (int64_t)s * p.drafts * draft_bytes + hk * (D * 2);
      }
      kr[i] = load_vec(static_cast<const char*>(p.k_pool) + (base + (pool ? 0 : k_far)) + off, 0);
      vr[i] = load_vec(static_cast<const char*>(p.v_pool) + (base + (pool ? 0 : v_far)) + off, 0);
    }
  };
  // What a token's chunks are exchanged by in LDS: K is read from 8 tokens' chunk j at once, V from 4 tokens' four neighbouring ones.
  const auto v_swap = [](int t) { return CPT == 16 ? (t & 3) << 2 : (t >> 1 & 1) << 2; };
  const auto stage = [&](int tile, int buf) __attribute__((always_inline)) {
    const int end = tile < cached ? len - tile * kTile : drafts;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int t = run_of(i) + t_lane;
      sk[buf][t * CPT + (c_of ^ (t & (CPT - 1)))] = kr[i];
      const uint32_t keep = t < end ? ~0u : 0u;  // junk V must not meet the zeros of its probabilities
      sv[buf][t * CPT + (c_of ^ v_swap(t))] = make_uint4(vr[i].x & keep, vr[i].y & keep, vr[i].z & keep, vr[i].w & keep);
    }
  };

  // The first two tiles' pages, and behind them the length that says whether there are such tiles.
  lookup(split);
  // ---- queries -----------------------------------------------------------------------------------------------------------
  const int num_q_heads = p.num_kv_heads * group;
  const int r = row0 + 32 * wave + n;  // (behind the last one: the first one again, and written nowhere)
  const int draft = r < rows ? r / group : 0, head = r < rows ? r - draft * group : 0;
  bf16x8_t q[CH];
  {
    const uint4* from = static_cast<const uint4*>(p.q) + (((int64_t)s * p.drafts + draft) * num_q_heads + hk * group + head) * CPT;
    // The largest product is to be the largest logit: a negative scale goes into the queries' signs, and one of zero makes them zeros.
    const uint32_t flip = p.scale_log2e < 0.f ? 0x80008000u : 0u, keep = p.scale_log2e != 0.f ? ~0u : 0u;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      uint4 v = from[2 * j + h];
      v.x = (v.x ^ flip) & keep, v.y = (v.y ^ flip) & keep, v.z = (v.z ^ flip) & keep, v.w = (v.w ^ flip) & keep;
      q[j] = __builtin_bit_cast(bf16x8_t, v);
    }
  }
  const float scale = p.scale_log2e != 0.f ? fabsf(p.scale_log2e) : 1.f;
  const uint64_t sees = p.mask[(int64_t)s * p.drafts + draft];  // (tokens behind the last draft are masked by their number)

  f32x16_t acc[E];
  float m_run = kNegInf, m_ref = 0.f, l_run = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;

  const bool works = row0 + 32 * wave < rows;  // (a wave without rows brings its runs all the same)
  // Tile i of this workgroup is number split + i * splits.  While one is computed, the next is in LDS (or on its way there) and the one behind
  // it in registers (or on its way there).
  const auto number = [&](int i) { return split + i * splits; };
  fetch(number(0));
  lookup(number(1));
  stage(number(0), 0);
  fetch(number(1));
  lookup(number(2));
  // Where a lane reads K, and V: each 16 lanes get 16 elements of four tokens, turned so that a lane has one element of the four.
  const int k_swap = h ^ (n & (CPT - 1));
  const int v_tok = 4 * h + (lane & 15) / 4;  // and 8 more for the other four, of every 16 tokens
  const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), v_half = lane & 1;
  uint32_t v_at[2][E];  // in 8 bytes
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int t = v_tok + 8 * b;
      v_at[b][e] = (uint32_t)(t * CPT + ((4 * e + v_chunk) ^ v_swap(t))) * 2u + (uint32_t)v_half;
    }
  const auto logits = [&](int buf, f32x16_t (&x)[2]) __attribute__((always_inline)) {
    const uint4* kt = &sk[buf][n * CPT];
    uint4 k[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) k[j] = kt[(2 * j) ^ k_swap];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        x[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[j]), q[j], j == 0 ? f32x16_t{} : x[sub], 0, 0, 0);
        if (sub == 0) k[j] = kt[32 * CPT + ((2 * j) ^ k_swap)];
      }
    }
  };
  const auto values = [&](int tile, int buf, f32x16_t (&x)[2]) __attribute__((always_inline)) {
    lds_s16x4_t* const vt = (lds_s16x4_t*)&sv[buf][0];
    const int end = tile < cached ? len - tile * kTile : drafts;
    if (end < kTile || tile >= cached) {
      const uint64_t mine = (tile < cached ? ~0ull : sees) >> (4 * h);
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = 32 * sub + 8 * (i / 4) + i % 4;  // and 4 h
          if (t + 4 * h >= end || ((mine >> t) & 1u) == 0) x[sub][i] = kNegInf;
        }
    }
    float mx = kNegInf;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[sub][i]);
    mx *= scale;
    if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0ull) {
      mx = halves_max(mx);
      const float m_new = mx > m_run ? mx + kGrow : m_run;
      const float ref = m_new == kNegInf ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - ref);
      l_run *= alpha;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= alpha;
      m_run = m_new;
      m_ref = ref;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {  // 16 tokens
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x[c / 2][8 * (c % 2) + 2 * i], scale, -m_ref));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(x[c / 2][8 * (c % 2) + 2 * i + 1], scale, -m_ref));
        const Terms t = terms_of(p0, p1);
        hi[i] = t.hi;
        lo[i] = t.lo;
        l_run += p0 + p1;
      }
      const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
      const bf16x8_t pl = __builtin_bit_cast(bf16x8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
      bf16x8_t v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vt + v_at[0][e] + c * 16 * CPT * 2);
        const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vt + v_at[1][e] + c * 16 * CPT * 2);
        v[e] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[e], ph, acc[e], 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[e], pl, acc[e], 0, 0, 0);
    }
  };
  // Tile i is in LDS half i % 2.
  const auto turn = [&](int i, auto parity) __attribute__((always_inline)) {
    constexpr int kNow = decltype(parity)::value, kNext = kNow ^ 1;
    __syncthreads();  // this tile is in LDS, and nobody reads the other half any more
    const bool real = works && number(i) < tiles;
    f32x16_t x[2];
    if (real) logits(kNow, x);
    stage(number(i + 1), kNext);
    fetch(number(i + 2));
    lookup(number(i + 3));
    if (real) values(number(i), kNow, x);
  };
  for (int i = 0; number(i) < tiles; i += 2) {  // (always both: on a way out between them the loads that are waited for next would be the last)
    turn(i, Parity<0>{});
    turn(i + 1, Parity<1>{});
  }

  // ---- every wave has its rows' whole states: lane (h, n) rows 8*(i/4) + 4*h + i%4 of C, elements 32*e + row of query n ---------------
  if (r >= rows) return;
  const float l = halves_sum(l_run);
  if (!several) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* out = static_cast<uint16_t*>(p.out) + (((int64_t)s * p.drafts + draft) * num_q_heads + hk * group + head) * D;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 2) store_pair<bf16_t>(out, (32 * e + 8 * (i / 4) + 4 * h + i % 4) / 2, acc[e][i] * inv, acc[e][i + 1] * inv);
  } else {
    float* record = p.partials + (slot * (p.drafts * group) + r) * (D + 2);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 2)
        *reinterpret_cast<float2*>(record + 32 * e + 8 * (i / 4) + 4 * h + i % 4) = make_float2(acc[e][i], acc[e][i + 1]);
    if (h == 0) *reinterpret_cast<float2*>(record + D) = make_float2(m_run, l);
  }
}

}  // namespace

hipError_t launch_tree_wide(const RowsArgs& a, RowsParams p, hipStream_t stream) {
  dim3 blocks;
  if (!rows_grid(a, kWideRows, &p, &blocks)) return hipErrorInvalidValue;
  if (a.head_dim == 64)
    hipLaunchKernelGGL((tree_wide_kernel<64>), blocks, dim3(NT), 0, stream, p);
  else
    hipLaunchKernelGGL((tree_wide_kernel<128>), blocks, dim3(NT), 0, stream, p);
  return hipGetLastError();
}

}  // namespace pe
