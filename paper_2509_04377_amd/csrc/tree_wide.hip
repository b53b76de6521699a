// Attention of a tree of drafted tokens over a paged bfloat16 cache, for many query rows: more than 32 share the K and V of a row.
//
// The products count here, not the traffic: 256 query rows ask for 256 operations a byte of the cache.  A workgroup owns 32 query rows a
// wave and one split of the tokens (tiles of 64, the drafts are the last one); K and V of a tile go through LDS once for all its waves,
// which read them as operands of the 32 x 32 x 16 products.  Two tiles are on their way to registers while one is computed out of one half
// of LDS and the next is put into the other; one barrier a tile.
//
// With lane l = 32*h + n:
//   QK (A = K, B = Q): C[m][n] = <k_m, q_n>.  Lane l reads 16 bytes of token n (as row m), chunk 2*j + h; a token's chunks lie in LDS in an
//   order of their own (chunk ^ token), so that neighbouring tokens' do not meet in the same banks.  Lane l is left with tokens
//   8*(i/4) + 4*h + i%4 of query n, i < 16.
//   PV (A = V transposed, B = P): a product contracts 16 tokens, lane half h those that it has: registers 8*c .. 8*c + 7 of the logits.  Row m
//   of A is d = m*E + e in product e, E = D/32: lane l reads elements n*E .. of its eight tokens, and byte permutes bring a token's
//   elements together with the others'.
//
// Probabilities go into the product as two bfloat16 terms, as in paged_rows.hip, and the softmax is that one too.
#include "pe_rows_device.h"

namespace pe {
namespace {

constexpr int kTile = 64;  // tokens

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

template <int P>
struct Parity {
  static constexpr int value = P;
};

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 2) void tree_wide_kernel(const RowsParams p) {
  constexpr int NT = WAVES * kWave, ROWS = 32 * WAVES;
  constexpr int CPT = D / 8;                 // 16-byte chunks of a token
  constexpr int NL = kTile * CPT / NT;       // 16-byte chunks of K (and of V) that a lane brings
  constexpr int CH = D / 16;                 // products of QK
  constexpr int E = D / 32;                  // elements of V that a lane reads of a token
  constexpr int SETS = WAVES == 8 ? 2 : 1;
  static_assert(NL * NT == kTile * CPT, "whole chunks");
  __shared__ uint4 sk[2][kTile * CPT], sv[2][kTile * CPT];

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int h = lane >> 5, n = lane & 31, tid = (int)threadIdx.x;
  const int log2_block = shape_log2_block(p.shape), group = shape_group(p.shape), splits = shape_splits(p.shape);
  const Place at = place_at(blockIdx.x, blockIdx.y, (p.shape & kShapeXcd) != 0, (p.shape & kShapeLinear) != 0, splits * p.tiles, p.num_kv_heads,
                            p.inv_heads);
  const int s = at.seq, hk = at.head, split = at.split / p.tiles, tile0 = at.split - split * p.tiles;
  const bool shared = p.max_blocks < 0;
  const int max_blocks = shared ? -p.max_blocks : p.max_blocks;
  // (read only while the launch runs: scalar loads, which the barriers would otherwise forbid)
  const auto* table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
      reinterpret_cast<uintptr_t>(p.block_table + (int64_t)(shared ? s : at.row) * max_blocks));
  const int drafts = drafts_of(p, s), rows = drafts * group, row0 = tile0 * ROWS;
  if (row0 >= rows) return;
  const int len = length_of(p, s, max_blocks, log2_block);
  const int cached = len / kTile + (len % kTile != 0), tiles = cached + 1;

  // ---- staging ------------------------------------------------------------------------------------------------------------
  // A wave brings NL runs of K and of V of a tile, TPL token rows each, which lie in one page: its place is looked up with scalar loads.
  constexpr int TPL = kWave / CPT;
  const int t_lane = lane / CPT, c_of = lane % CPT;
  const uint32_t token_bytes = (uint32_t)(shared ? p.num_kv_heads : 1) * (D * 2), draft_bytes = (uint32_t)p.num_kv_heads * (D * 2);
  const uint32_t lane_off = (uint32_t)t_lane * token_bytes + (uint32_t)c_of * 16u;
  const auto run_of = [&](int i) { return (i * WAVES + wave) * TPL; };  // the first token of run i in its tile
  int ids[NL];
  const auto lookup = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int64_t j = ((int64_t)tile * kTile + run_of(i)) >> log2_block;
      ids[i] = table[j < max_blocks ? (int)j : max_blocks - 1];
    }
  };
  // With eight waves two tiles are on their way, each set of registers belongs to every other tile of this workgroup; fewer waves have as
  // many bytes on their way with one.
  uint4 kr[SETS][NL], vr[SETS][NL];
  const auto fetch = [&](int tile, uint4 (&k)[NL], uint4 (&v)[NL]) __attribute__((always_inline)) {  // (what is no token, or no tile, reads one that is)
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
      k[i] = load_vec(static_cast<const char*>(pool ? p.k_pool : p.k_draft) + base + off, 0);
      v[i] = load_vec(static_cast<const char*>(pool ? p.v_pool : p.v_draft) + base + off, 0);
    }
  };
  const auto stage = [&](int tile, int buf, const uint4 (&k)[NL], const uint4 (&v)[NL]) __attribute__((always_inline)) {
    const int end = tile < cached ? len - tile * kTile : drafts;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int t = run_of(i) + t_lane;
      sk[buf][t * CPT + (c_of ^ (t & (CPT - 1)))] = k[i];
      const uint32_t keep = t < end ? ~0u : 0u;  // junk V must not meet the zeros of its probabilities
      sv[buf][t * CPT + c_of] = make_uint4(v[i].x & keep, v[i].y & keep, v[i].z & keep, v[i].w & keep);
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
  fetch(number(0), kr[0], vr[0]);
  lookup(number(1));
  if constexpr (SETS == 2) {
    fetch(number(1), kr[1], vr[1]);
    lookup(number(2));
  }
  stage(number(0), 0, kr[0], vr[0]);
  fetch(number(SETS), kr[0], vr[0]);
  lookup(number(SETS + 1));
  const auto compute = [&](int tile, int buf) __attribute__((always_inline)) {
    const uint4* kt = &sk[buf][n * CPT];
    const uint32_t* vt = reinterpret_cast<const uint32_t*>(&sv[buf][0]) + 4 * h * (D / 2) + n * (E / 2);
    const int end = tile < cached ? len - tile * kTile : drafts;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {  // 32 tokens
      f32x16_t x;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const uint4 k = kt[sub * 32 * CPT + ((2 * j) ^ (h ^ (n & (CPT - 1))))];
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), q[j], x, 0, 0, 0);
      }
      if (end < kTile || tile >= cached) {
        const uint64_t mine = (tile < cached ? ~0ull : sees) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = 32 * sub + 8 * (i / 4) + i % 4;  // and 4 h
          if (t + 4 * h >= end || ((mine >> t) & 1u) == 0) x[i] = kNegInf;
        }
      }
      float mx = kNegInf;
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[i]);
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
      for (int c = 0; c < 2; ++c) {  // 16 tokens
        float pr[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) pr[i] = __builtin_amdgcn_exp2f(fmaf(x[8 * c + i], scale, -m_ref));
        l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t p0 = __float_as_uint(pr[2 * w]), p1 = __float_as_uint(pr[2 * w + 1]);
          hw[w] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
          const float r0 = pr[2 * w] - __uint_as_float(p0 & 0xffff0000u), r1 = pr[2 * w + 1] - __uint_as_float(p1 & 0xffff0000u);
          lw[w] = __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x07060302u);
        }
        const bf16x8_t hi = __builtin_bit_cast(bf16x8_t, make_uint4(hw[0], hw[1], hw[2], hw[3]));
        const bf16x8_t lo = __builtin_bit_cast(bf16x8_t, make_uint4(lw[0], lw[1], lw[2], lw[3]));
        uint32_t vb[8][E / 2];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const uint32_t* from = vt + (32 * sub + 16 * c + (t / 4) * 8 + t % 4) * (D / 2);
          if constexpr (E == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(from);
            vb[t][0] = v.x, vb[t][1] = v.y;
          } else {
            vb[t][0] = from[0];
          }
        }
        bf16x8_t va[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
          va[e] = __builtin_bit_cast(bf16x8_t, make_uint4(__builtin_amdgcn_perm(vb[1][e >> 1], vb[0][e >> 1], sel),
                                                          __builtin_amdgcn_perm(vb[3][e >> 1], vb[2][e >> 1], sel),
                                                          __builtin_amdgcn_perm(vb[5][e >> 1], vb[4][e >> 1], sel),
                                                          __builtin_amdgcn_perm(vb[7][e >> 1], vb[6][e >> 1], sel)));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[e], hi, acc[e], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[e], lo, acc[e], 0, 0, 0);
      }
    }
  };
  // Tile i is in LDS half i % 2 and was in registers i % SETS.
  const auto turn = [&](int i, auto parity) __attribute__((always_inline)) {
    constexpr int kNow = decltype(parity)::value, kNext = kNow ^ 1, kSet = kNext % SETS;
    __syncthreads();  // this tile is in LDS, and nobody reads the other half any more
    stage(number(i + 1), kNext, kr[kSet], vr[kSet]);
    fetch(number(i + 1 + SETS), kr[kSet], vr[kSet]);
    lookup(number(i + 2 + SETS));
    if (works && number(i) < tiles) compute(number(i), kNow);
  };
  for (int i = 0; number(i) < tiles; i += 2) {  // (always both: on a way out between them the loads that are waited for next would be the last)
    turn(i, Parity<0>{});
    turn(i + 1, Parity<1>{});
  }

  // ---- every wave has its rows' whole states: lane (h, n) rows m = 8*(i/4) + 4*h + i%4 of C, elements m*E + e of query n ------------
  if (r >= rows) return;
  const float l = halves_sum(l_run);
  if (splits == 1) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint32_t* out = static_cast<uint32_t*>(p.out) + (((int64_t)s * p.drafts + draft) * num_q_heads + hk * group + head) * (D / 2);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int m = 8 * (i / 4) + 4 * h + i % 4;
      uint32_t w[E / 2];
#pragma unroll
      for (int e = 0; e < E; e += 2)
        w[e / 2] = (uint32_t)f32_to_bf16(acc[e][i] * inv) | ((uint32_t)f32_to_bf16(acc[e + 1][i] * inv) << 16);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) out[m * (E / 2) + e] = w[e];
    }
  } else {
    float* record = p.partials + (((int64_t)at.row * splits + split) * (p.drafts * group) + r) * (D + 2);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int m = 8 * (i / 4) + 4 * h + i % 4;
#pragma unroll
      for (int e = 0; e < E; e += 2) *reinterpret_cast<float2*>(record + m * E + e) = make_float2(acc[e][i], acc[e + 1][i]);
    }
    if (h == 0) *reinterpret_cast<float2*>(record + D) = make_float2(m_run, l);
  }
}

template <int D>
hipError_t launch_wide(const RowsArgs& a, RowsParams p, hipStream_t stream) {
  dim3 blocks;
  if (!rows_grid(a, a.tile_rows, &p, &blocks)) return hipErrorInvalidValue;
  if (a.tile_rows == 64)
    hipLaunchKernelGGL((tree_wide_kernel<D, 2>), blocks, dim3(2 * kWave), 0, stream, p);
  else if (a.tile_rows == 128)
    hipLaunchKernelGGL((tree_wide_kernel<D, 4>), blocks, dim3(4 * kWave), 0, stream, p);
  else if (a.tile_rows == 256)
    hipLaunchKernelGGL((tree_wide_kernel<D, 8>), blocks, dim3(8 * kWave), 0, stream, p);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_wide(const RowsArgs& a, const RowsParams& p, hipStream_t stream) {
  return a.head_dim == 64 ? launch_wide<64>(a, p, stream) : launch_wide<128>(a, p, stream);
}

}  // namespace pe
