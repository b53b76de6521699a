// Paged decode attention over a cache in 8 bits (pe_quant_decode): QK and PV on the matrix cores in bfloat16, which holds every e4m3 number.
//
// The work is cut, and the products are laid out, as in paged_decode_bf16.hip (which explains the index maps): a workgroup owns one split of
// one (sequence, KV head) row, whose 16-token tiles are dealt out to splits and waves round robin; lane l = 16 g + m holds eight elements of a
// token, here 8 bytes, which become the 16 bytes of an operand by four conversions.  A tile lies in one page: its logits take K's scale
// of that page, its softmax weights V's on their way into the product with V.
//
//   QK   16x16x32; fp32 queries enter as three bfloat16 terms, which hold all of their bits, in one chain of products.
//   PV   16x16x16; the four lanes of a quad hold the same weight and feed one term of its exact decomposition into three each.
//
// The tokens behind the last full page lie in the row's tail in the activations' type.  They are further tiles of the same kind that come
// without conversion (bfloat16) or as three terms (fp32: products of terms below 2^-24 of the whole are left out), with a scale of 1.  A
// wave's first one is asked for in front of its other tiles and taken behind them.
#include "pe_decode_common.h"
#include "pe_quant.h"

namespace pe {
namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kGrow = 3.f;  // how far above the largest logit (log2) the softmax reference is set
constexpr int kTile = 16;     // tokens

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

template <int CTRL>
__device__ __forceinline__ float quad_perm_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float v) { return quad_perm_add<0x4E>(quad_perm_add<0xB1>(v)); }

// Element c (0..3) of a vector, c per lane: b0 = c & 1, b1 = c & 2.
__device__ __forceinline__ float pick4(const f32x4_t& v, bool b0, bool b1) {
  const float lo = b0 ? v[1] : v[0];
  const float hi = b0 ? v[3] : v[2];
  return b1 ? hi : lo;
}

// Two e4m3 numbers (the lower or the upper half of a word) as two bfloat16.
template <bool UPPER>
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, UPPER));
}
__device__ __forceinline__ u32x4_t widen8(const u32x2_t& w) {
  return u32x4_t{widen2<false>(w[0]), widen2<true>(w[0]), widen2<false>(w[1]), widen2<true>(w[1])};
}

// Eight elements in the activations' type as bfloat16 operands: one, or three whose sum they are (each what a truncation leaves of the rest).
template <typename T>
struct Terms;
template <>
struct Terms<bf16_t> {
  static constexpr int N = 1;
  static constexpr int kVecs = 1;  // 16-byte vectors of eight elements
  static __device__ __forceinline__ void split(const u32x4_t (&raw)[1], u32x4_t (&t)[1]) { t[0] = raw[0]; }
};
template <>
struct Terms<float> {
  static constexpr int N = 3;
  static constexpr int kVecs = 2;
  static __device__ __forceinline__ void split(const u32x4_t (&raw)[2], u32x4_t (&t)[3]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = __uint_as_float(raw[i / 2][i % 2 * 2]), b = __uint_as_float(raw[i / 2][i % 2 * 2 + 1]);
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        const uint32_t ha = __float_as_uint(a), hb = __float_as_uint(b);
        t[n][i] = __builtin_amdgcn_perm(hb, ha, 0x07060302u);
        a -= __uint_as_float(ha & 0xffff0000u);
        b -= __uint_as_float(hb & 0xffff0000u);
      }
    }
  }
};

struct QuantParams {
  const void* q;
  const void* k_tail;
  const void* v_tail;
  void* out;
  float* partials;
  uint64_t tag;
  float scale_log2e;
};

// One wave's view of a tile.  HG: groups of four query heads (G <= 4: 1, G <= 8: 2).
template <typename T, int D, int HG>
struct Tile {
  static constexpr int LPR = D / 8;
  static constexpr int TPL = kWave / LPR;
  static constexpr int NL = kTile / TPL;
  static constexpr int NT = 4 / NL;  // tokens that a row of the K operand carries (1 or 2)
  static constexpr int NQ = Terms<T>::N;

  int g;
  bool b0, b1;                   // bits of the class c = lane & 3
  uint32_t term1, term2, term3;  // all ones in the upper half for classes >= 1, 2, 3
  uint32_t sel_even, sel_odd;    // D = 64: byte selectors that put an element into its parity's place

  __device__ __forceinline__ int token_of(int j) const { return TPL * (j / NT) + NT * g + j % NT; }

  // The part of the tile's logits that K's term `k` gives with the queries' first `terms` terms, added to c.
  template <int TERMS>
  __device__ __forceinline__ void products(const u32x4_t (&k)[NL], const bf16x8_t (&qop)[NQ][HG][NT], f32x4_t (&c)[HG][4]) const {
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
      for (int hg = 0; hg < HG; ++hg)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int n = 0; n < TERMS; ++n)
            c[hg][i * NT + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[i]), qop[n][hg][t], c[hg][i * NT + t], 0, 0, 0);
  }

  static __device__ __forceinline__ void regrow(float mx, float& m_run, float& m_ref, float& l_run, f32x4_t (&acc)[8]) {
    mx = rows_max(mx);
    const float m_new = mx > m_run ? mx + kGrow : m_run;
    const float ref = m_new == kNegInf ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - ref);
    l_run *= alpha;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= alpha;
    m_run = m_new;
    m_ref = ref;
  }

  // Softmax weights of this lane's four tokens, their sum, and the operand of PV: the weights times V's scale.
  __device__ __forceinline__ s16x4_t probs(const float (&x)[4], float m_ref, float v_scale, float& l_run) const {
    uint32_t t[4];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float p = __builtin_amdgcn_exp2f(x[j] - m_ref);
      sum += p;
      p *= v_scale;
      p -= __uint_as_float(__float_as_uint(p) & term1);
      p -= __uint_as_float(__float_as_uint(p) & term2);
      p -= __uint_as_float(__float_as_uint(p) & term3);
      t[j] = __float_as_uint(p);
    }
    l_run += sum;
    const u32x2_t packed = {__builtin_amdgcn_perm(t[1], t[0], 0x07060302u), __builtin_amdgcn_perm(t[3], t[2], 0x07060302u)};
    return __builtin_bit_cast(s16x4_t, packed);
  }

  __device__ __forceinline__ s16x4_t v_operand(const u32x4_t (&vb)[NL], int e) const {
    u32x2_t a;
    if constexpr (D == 128) {
      const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
      a[0] = __builtin_amdgcn_perm(vb[1][e >> 1], vb[0][e >> 1], sel);
      a[1] = __builtin_amdgcn_perm(vb[3][e >> 1], vb[2][e >> 1], sel);
    } else {
      const uint32_t sel = (e & 1) ? sel_odd : sel_even;
      a[0] = __builtin_amdgcn_perm(0u, vb[0][e >> 1], sel);
      a[1] = __builtin_amdgcn_perm(0u, vb[1][e >> 1], sel);
    }
    return __builtin_bit_cast(s16x4_t, a);
  }
  __device__ __forceinline__ void accumulate(const u32x4_t (&vb)[NL], const s16x4_t (&pop)[HG], f32x4_t (&acc)[HG][8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const s16x4_t a = v_operand(vb, e);
#pragma unroll
      for (int hg = 0; hg < HG; ++hg) acc[hg][e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, pop[hg], acc[hg][e], 0, 0, 0);
    }
  }
};

template <typename T, int D, int HG, int WAVES, int DEPTH, bool SHARED, bool TAGGED>
__global__ __launch_bounds__(WAVES * kWave, 2) void quant_decode_kernel(
    const int32_t* seq_lens, const int32_t* block_table, const void* k_pool, const void* v_pool, const float* scales,
    const int num_kv_heads, const int max_blocks, const uint32_t inv_heads, const uint32_t shape, const QuantParams p) {
  using TL = Tile<T, D, HG>;
  constexpr int LPR = TL::LPR, TPL = TL::TPL, NL = TL::NL, NT = TL::NT, NQ = TL::NQ, NV = Terms<T>::kVecs;
  constexpr int GH = 4 * HG;  // heads computed; g_real of them exist

  __shared__ WaveStates<WAVES, GH, D> sm;

  const int log2_block = shape_log2_block(shape), g_real = shape_group(shape), splits = shape_splits(shape);
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int g = lane >> 4, m = lane & 15, c = lane & 3;
  const Place at = decode_place(shape, num_kv_heads, inv_heads);
  const int row = at.row, split = at.split, s = at.seq, hk = at.head;
  const int32_t* bt = block_table + (int64_t)(SHARED ? s : row) * max_blocks;
  const int stride = splits * WAVES, first = split * WAVES + wave;
  const int tiles_log2 = log2_block - ilog2(kTile), in_page = (1 << tiles_log2) - 1;

  // (an unused entry, -1, is replaced by page 0: its tokens are masked, so any address inside the pool will do)
  const auto lookup = [&](int tile) {
    int pi = tile >> tiles_log2;
    pi = pi < max_blocks ? pi : max_blocks - 1;
    const int ph = __builtin_amdgcn_readfirstlane(bt[pi]);
    return ph < 0 ? 0 : ph;
  };
  int phys[DEPTH + 1];
#pragma unroll
  for (int d = 0; d <= DEPTH; ++d) phys[d] = lookup(first + d * stride);
  const int len_raw = seq_lens[s];
  __builtin_amdgcn_sched_barrier(0);

  TL tl;
  tl.g = g;
  tl.b0 = (c & 1) != 0;
  tl.b1 = (c & 2) != 0;
  tl.term1 = c >= 1 ? 0xffff0000u : 0u;
  tl.term2 = c >= 2 ? 0xffff0000u : 0u;
  tl.term3 = c >= 3 ? 0xffff0000u : 0u;
  const bool tp = m >= 8;
  tl.sel_even = tp ? 0x01000c0cu : 0x0c0c0100u;
  tl.sel_odd = tp ? 0x03020c0cu : 0x0c0c0302u;
  const int block = D == 128 ? g : (g & 1);
  const int k_slice = 4 * block + c, v_slice = lane % LPR;
  const int k_tok = D == 128 ? (m >> 2) : 2 * (m >> 2) + (g >> 1), v_tok = lane / LPR;
  const int row_vecs = SHARED ? LPR * num_kv_heads : LPR;  // slices between consecutive tokens of this head
  const int head_vecs = SHARED ? hk * LPR : 0;
  const int k_off = k_tok * row_vecs + head_vecs + k_slice, v_off = v_tok * row_vecs + head_vecs + v_slice;

  const int most = max_blocks << log2_block;  // (a longer length is a caller error: the table row is the end)
  const int len = len_raw < 0 ? 0 : len_raw < most || most <= 0 ? len_raw : most;
  const int full = len >> log2_block << log2_block;  // tokens in 8 bits
  const int ntiles = full >> ilog2(kTile), tail_tiles = (len - full + kTile - 1) >> ilog2(kTile);

  float m_run[HG], m_ref[HG], l_run[HG];
  f32x4_t acc[HG][8];
#pragma unroll
  for (int hg = 0; hg < HG; ++hg) {
    m_run[hg] = kNegInf;
    m_ref[hg] = 0.f;
    l_run[hg] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[hg][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // The tail's tiles go on where those of the full pages end, as if they were dealt out together.
  if (first < ntiles + tail_tiles) {
    const auto base_of = [&](int tile, int ph) { return (((int64_t)ph << log2_block) + ((tile & in_page) * kTile)) * row_vecs; };
    const auto issue = [&](u32x2_t(&buf)[NL], const void* pool, int64_t base, int off) {
#pragma unroll
      for (int i = 0; i < NL; ++i) buf[i] = __builtin_nontemporal_load(static_cast<const u32x2_t*>(pool) + base + (int64_t)i * TPL * row_vecs + off);
    };
    const auto scales_of = [&](int ph) {
      const float* at = scales + ((int64_t)ph * (SHARED ? num_kv_heads : 1) + (SHARED ? hk : 0)) * 2;
      return make_float2(at[0], at[1]);
    };
    u32x2_t kb[DEPTH][NL], vb[DEPTH][NL];
    float2 sc[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const bool more = first + d * stride < ntiles;
      const int64_t there = base_of(first + d * stride, phys[d]), base = more ? there : 0;
      issue(kb[d], k_pool, base, more ? k_off : 0);
      issue(vb[d], v_pool, base, more ? v_off : 0);
      sc[d] = scales_of(more ? phys[d] : 0);
    }
    // queries: column n = 4 h + c of the operand holds the class-c slices of head h
    bf16x8_t qop[NQ][HG][NT];
#pragma unroll
    for (int hg = 0; hg < HG; ++hg) {
      const int h = 4 * hg + (m >> 2);
      const int64_t head = (int64_t)s * num_kv_heads * g_real + hk * g_real + (h < g_real ? h : 0);
      u32x4_t raw[NV], t[NQ];
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = static_cast<const u32x4_t*>(p.q)[(head * LPR + k_slice) * NV + i];
      Terms<T>::split(raw, t);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const u32x4_t zero = {0u, 0u, 0u, 0u};
          const bool in = h < g_real && (NT == 1 || (g >> 1) == nt);
          qop[n][hg][nt] = __builtin_bit_cast(bf16x8_t, in ? t[n] : zero);
        }
    }

    // From a tile's products to its part of the sums; `left` of its tokens exist.
    const auto softmax = [&](const f32x4_t(&prod)[HG][4], float k_scale, float v_scale, int left, s16x4_t(&pop)[HG]) {
      float x[HG][4], mx[HG];
      bool grow = false;
#pragma unroll
      for (int hg = 0; hg < HG; ++hg) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[hg][j] = quad_sum(pick4(prod[hg][j], tl.b0, tl.b1)) * k_scale;
          if (left < kTile) x[hg][j] = tl.token_of(j) < left ? x[hg][j] : kNegInf;
        }
        mx[hg] = fmaxf(fmaxf(x[hg][0], x[hg][1]), fmaxf(x[hg][2], x[hg][3]));
        grow = grow || mx[hg] > m_run[hg];
      }
      if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) TL::regrow(mx[hg], m_run[hg], m_ref[hg], l_run[hg], acc[hg]);
      }
#pragma unroll
      for (int hg = 0; hg < HG; ++hg) pop[hg] = tl.probs(x[hg], m_ref[hg], v_scale, l_run[hg]);
    };

    int ph_next = phys[DEPTH];
    int tile0 = first;
    for (; tile0 < ntiles; tile0 += DEPTH * stride) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int tile = tile0 + d * stride;  // past the end (an odd last one): every token is masked
        const int left = tile < ntiles ? kTile : 0;
        f32x4_t prod[HG][4];
#pragma unroll
        for (int hg = 0; hg < HG; ++hg)
#pragma unroll
          for (int j = 0; j < 4; ++j) prod[hg][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        u32x4_t op[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) op[i] = widen8(kb[d][i]);
        tl.template products<NQ>(op, qop, prod);
        const int ahead = tile + DEPTH * stride;
        const bool more = ahead < ntiles;
        const int64_t there = base_of(ahead, ph_next), base = more ? there : 0;
        const float2 now = sc[d];
        sc[d] = scales_of(more ? ph_next : 0);
        ph_next = lookup(ahead + stride);
        issue(kb[d], k_pool, base, more ? k_off : 0);
        s16x4_t pop[HG];
        softmax(prod, now.x * p.scale_log2e, left ? now.y : 0.f, left, pop);
#pragma unroll
        for (int i = 0; i < NL; ++i) op[i] = widen8(left ? vb[d][i] : u32x2_t{0u, 0u});
        tl.accumulate(op, pop, acc);
        issue(vb[d], v_pool, base, more ? v_off : 0);
      }
    }

    while (tile0 - stride >= ntiles && tile0 > first) tile0 -= stride;
    for (int tail = tile0 - ntiles; tail < tail_tiles; tail += stride) {
      const int tok0 = tail * kTile, left = len - full - tok0;
      // [S][Hk][B][D] in either layout
      const u32x4_t* kt = static_cast<const u32x4_t*>(p.k_tail) + (((int64_t)row << log2_block) + tok0) * (LPR * NV);
      const u32x4_t* vt = static_cast<const u32x4_t*>(p.v_tail) + (((int64_t)row << log2_block) + tok0) * (LPR * NV);
      u32x4_t kterm[NQ][NL], vterm[NQ][NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        u32x4_t raw[NV], t[NQ];
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = kt[((TPL * i + k_tok) * LPR + k_slice) * NV + j];
        if (TPL * i + k_tok >= left) {  // what is no token must not meet its neighbour's zeros (0 * NaN)
#pragma unroll
          for (int j = 0; j < NV; ++j) raw[j] = u32x4_t{0u, 0u, 0u, 0u};
        }
        Terms<T>::split(raw, t);
#pragma unroll
        for (int n = 0; n < NQ; ++n) kterm[n][i] = t[n];
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = vt[((TPL * i + v_tok) * LPR + v_slice) * NV + j];
        if (TPL * i + v_tok >= left) {
#pragma unroll
          for (int j = 0; j < NV; ++j) raw[j] = u32x4_t{0u, 0u, 0u, 0u};
        }
        Terms<T>::split(raw, t);
#pragma unroll
        for (int n = 0; n < NQ; ++n) vterm[n][i] = t[n];
      }
      f32x4_t prod[HG][4];
#pragma unroll
      for (int hg = 0; hg < HG; ++hg)
#pragma unroll
        for (int j = 0; j < 4; ++j) prod[hg][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      tl.template products<NQ>(kterm[0], qop, prod);
      if constexpr (NQ == 3) {
        tl.template products<3>(kterm[1], qop, prod);
        tl.template products<2>(kterm[2], qop, prod);  // (the third terms' product is below 2^-28 of the whole)
      }
      s16x4_t pop[HG];
      softmax(prod, p.scale_log2e, 1.f, left < kTile ? left : kTile, pop);
#pragma unroll
      for (int n = 0; n < NQ; ++n) tl.accumulate(vterm[n], pop, acc);
    }
    // (the placeholder loads behind a wave's last tiles: their registers are in use until they are back)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
#pragma unroll
      for (int i = 0; i < NL; ++i) asm volatile("" : : "v"(kb[d][i]), "v"(vb[d][i]));
  }

  // ---- merge: columns of a quad, lane groups, then the waves through LDS -------------------------------
#pragma unroll
  for (int hg = 0; hg < HG; ++hg) {
    const float l = rows_sum(l_run[hg]);
    const int h = 4 * hg + (m >> 2);
    if (g == 0 && c == 0) sm.ml[wave][h] = make_float2(m_run[hg], l);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f32x4_t a = acc[hg][e];
#pragma unroll
      for (int r = 0; r < 4; ++r) a[r] = quad_sum(a[r]);
      o[e] = pick4(a, tl.b0, tl.b1);
      if constexpr (D == 64) o[e] = halves_sum(o[e]);  // the two token parities
    }
    if (D == 128 || g < 2) {
      float4* dst = reinterpret_cast<float4*>(&sm.acc[wave][h][(4 * g + c) * 8]);
      dst[0] = make_float4(o[0], o[1], o[2], o[3]);
      dst[1] = make_float4(o[4], o[5], o[6], o[7]);
    }
  }
  __syncthreads();
  DecodeParams dp{};
  dp.out = p.out;
  dp.partials = p.partials;
  dp.tag = p.tag;
  if constexpr (TAGGED)
    merge_arrived<T, true>(sm, dp, row, split, splits, g_real);
  else
    merge_waves<T>(sm, dp, row, split, splits, g_real);
}

using QuantKernel = void (*)(const int32_t*, const int32_t*, const void*, const void*, const float*, int, int, uint32_t, uint32_t, QuantParams);

template <typename T, int D, int HG, int WAVES, int DEPTH>
hipError_t launch_one(const QuantDecodeArgs& a, hipStream_t stream) {
  PlaceGrid grid;
  if (!place_grid(a.num_seqs, a.num_kv_heads, a.splits, true, &grid)) return hipErrorInvalidValue;
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const uint32_t shape = (uint32_t)log2_block | (uint32_t)(a.num_q_heads / a.num_kv_heads) << 3 | (grid.xcd ? kShapeXcd : 0u) |
                         (grid.linear ? kShapeLinear : 0u) | (uint32_t)a.splits << 9;
  QuantKernel kernel = a.shared ? quant_decode_kernel<T, D, HG, WAVES, DEPTH, true, false> : quant_decode_kernel<T, D, HG, WAVES, DEPTH, false, false>;
  if (a.tagged) {
    if constexpr (one_part_a_wave<4 * HG, D, WAVES>)
      kernel = a.shared ? quant_decode_kernel<T, D, HG, WAVES, DEPTH, true, true> : quant_decode_kernel<T, D, HG, WAVES, DEPTH, false, true>;
    else
      return hipErrorInvalidValue;
  }
  const QuantParams p{a.q, a.cache.k_tail, a.cache.v_tail, a.out, a.partials, a.tag, a.scale * 1.4426950408889634f};
  hipLaunchKernelGGL(kernel, dim3(grid.x, grid.y), dim3(WAVES * kWave), 0, stream, a.seq_lens, a.block_table, a.cache.k, a.cache.v, a.cache.scales,
                     a.num_kv_heads, a.max_blocks, grid.inv_heads, shape, p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_shape(const QuantDecodeArgs& a, hipStream_t stream) {
  const bool wide = a.num_q_heads / a.num_kv_heads > 4;
  if (a.waves == 8) return wide ? launch_one<T, D, 2, 8, 2>(a, stream) : launch_one<T, D, 1, 8, 2>(a, stream);
  return wide ? launch_one<T, D, 2, 4, 2>(a, stream) : launch_one<T, D, 1, 4, 2>(a, stream);
}

}  // namespace

hipError_t launch_quant_decode(const QuantDecodeArgs& a, hipStream_t stream) {
  hipError_t e = hipErrorInvalidValue;
  if (a.head_dim == 64) e = a.is_bf16 ? launch_shape<bf16_t, 64>(a, stream) : launch_shape<float, 64>(a, stream);
  if (a.head_dim == 128) e = a.is_bf16 ? launch_shape<bf16_t, 128>(a, stream) : launch_shape<float, 128>(a, stream);
  if (e != hipSuccess || a.splits == 1 || a.tagged) return e;
  DecodeArgs m{};
  m.out = a.out;
  m.partials = a.partials;
  m.num_seqs = a.num_seqs;
  m.num_kv_heads = a.num_kv_heads;
  m.num_q_heads = a.num_q_heads;
  m.head_dim = a.head_dim;
  m.splits = a.splits;
  m.xcd_map = 1;
  m.is_bf16 = a.is_bf16;
  return launch_decode_merge(m, stream);
}

}  // namespace pe
