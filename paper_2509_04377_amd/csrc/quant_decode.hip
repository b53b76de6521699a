// Paged decode attention over a cache in 8 bits (pe_quant_decode): QK and PV on the matrix cores in bfloat16, which holds every e4m3 number.
//
// A workgroup owns one split of one (sequence, KV head) row.  The row's 16-token tiles are dealt out round robin, tile t to split
// (t / WAVES) % splits, wave t % WAVES, so that a wave's first tile does not depend on the row's length; a tile lies in one page.  K and V go from
// memory to registers, from there through a conversion (two numbers an instruction) into the matrix instructions; nothing is staged in LDS.
//
// Lane l = 16 g + m.  The row's query heads have GW of the 16 columns each, head m / GW, class m % GW: four columns with up to four heads, two
// with up to eight.
//
//   QK (16x16x32; A = K, B = queries).  A wave-load is 1 KiB in a row, 16 bytes a lane (two operands of eight elements), 64 bytes of a row of A.
//   D = 64: that is a token, row m being token 4 (m % 4) + m / 4, and C[token][column] is a logit.  D = 128: half a token, load j, row m
//   being half m % 2 of token 8 j + 4 (m / 2 % 2) + m / 4, and column (head, class) has the queries' half class % 2, so that a logit
//   is the sum of two entries of C: a select and an add across neighbouring lanes.  (Without halves, two loads of 64 bytes of each of 16
//   tokens, the products need neither, but every 128-byte line is asked for twice: 256 rows x 2048 22.6 us.)  Either way lane l ends with
//   the logits of tokens 4 i + g, i < 4, for its head, the same in the GW lanes of it.  fp32 queries enter as three bfloat16 terms,
//   which hold all of their bits, in one chain of products.
//
//   PV (16x16x16; A = V transposed, B = weights): lane l holds elements EV m .. EV m + EV - 1 of tokens 4 i + g (EV = D / 16); element e of the
//   four, brought together by byte permutes in front of the conversion, is a column of A whose contraction index is the token order in
//   which the lane holds its weights, which are the other operand as they stand.  The classes of a head feed the terms of its weights:
//   bfloat16: two, rounded, which are the weight to within 2^-17 (with the first one cut off 2^-16, in as much time); fp32: three, which are all
//   of it (with two classes in two turns).
//
// A page's K scale goes to the logits, V's to the weights on their way into the product.  Softmax: online, base 2, one reference a head and
// wave, set kGrow above the largest logit and moved only when one exceeds it, so that rescaling and the exchange between lanes are rare.
//
// The tokens behind the last full page lie in the row's tail in the activations' type.  They are further tiles, which need no conversion
// (bfloat16) or come as three terms (fp32: of the nine products of terms the last, below 2^-28 of the whole, is left out), with scales of 1.
// They are dealt out from the other end, to the waves that have the fewest others, and taken first, while the first 8-bit tiles are on
// their way (behind them a wave waits for memory once more).
//
// Bound by memory, short rows by the chain of a launch.  256 rows of D = 128 x 2048, 135 MB: 21.3 us where the caches hold them (6.3 TB/s; the vector units issue in 41 % of
// the cycles), 24.8 from memory (5.4 TB/s); 32 rows x 65536, 516 MB: 80 us, 84 from memory (6.1 to 6.4 TB/s); 64 rows of D = 64 x 1024, 8.5 MB: 5.5 us.
#include "pe_decode_common.h"
#include "pe_quant.h"

namespace pe {
namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kGrow = 3.f;  // how far above the largest logit (log2) the softmax reference is set
constexpr int kTile = 16;     // tokens
constexpr int kMostBlock = 128;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

template <int CTRL>
__device__ __forceinline__ float quad_perm_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over the classes of a head, in every lane of it.
template <int GW>
__device__ __forceinline__ float class_sum(float v) {
  v = quad_perm_add<0xB1>(v);
  return GW == 4 ? quad_perm_add<0x4E>(v) : v;
}

// Two e4m3 numbers (the lower or the upper half of a word) as two bfloat16.
template <bool UPPER>
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, UPPER));
}

// Elements in the activations' type as bfloat16 operands: one, or three whose sum they are (each what a truncation leaves of the rest), made
// one after the other, so that a term's registers are free for the next.
template <typename T>
struct Terms;
template <>
struct Terms<bf16_t> {
  static constexpr int N = 1;
  static constexpr int kWords = 1;  // registers of two elements
  template <int E>
  static __device__ __forceinline__ void load(const void* from, int64_t element, uint32_t (&raw)[E / 2]) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(from) + element);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) raw[i] = w[i];
  }
  template <int E>
  static __device__ __forceinline__ void take(uint32_t (&raw)[E / 2], uint32_t (&t)[E / 2]) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) t[i] = raw[i];
  }
};
template <>
struct Terms<float> {
  static constexpr int N = 3;
  static constexpr int kWords = 2;
  template <int E>
  static __device__ __forceinline__ void load(const void* from, int64_t element, uint32_t (&raw)[E]) {
    const uint32_t* w = static_cast<const uint32_t*>(from) + element;
#pragma unroll
    for (int i = 0; i < E; ++i) raw[i] = w[i];
  }
  // The next term, and what is left without it.
  template <int E>
  static __device__ __forceinline__ void take(uint32_t (&raw)[E], uint32_t (&t)[E / 2]) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const uint32_t a = raw[2 * i], b = raw[2 * i + 1];
      t[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      raw[2 * i] = __float_as_uint(__uint_as_float(a) - __uint_as_float(a & 0xffff0000u));
      raw[2 * i + 1] = __float_as_uint(__uint_as_float(b) - __uint_as_float(b & 0xffff0000u));
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

// One wave's view of a tile.
template <typename T, int D, int GW>
struct Tile {
  static constexpr int NJ = D / 64;  // 16-byte loads of K, and parts of a token
  static constexpr int EV = D / 16;  // elements of V a lane and token
  static constexpr int NQ = Terms<T>::N;
  static constexpr int kTurns = NQ == 3 && GW == 2 ? 2 : 1;  // of PV
  typedef uint32_t VLoad __attribute__((ext_vector_type(EV / 4)));

  uint32_t cut;    // all ones in the upper half for classes that take a second or third term ..
  uint32_t cut2;   // .. a third
  float unit;      // 0 for classes without a term
  float l_run, m_run, m_ref;
  f32x4_t acc[EV];

  __device__ __forceinline__ void begin(int c) {
    if constexpr (NQ == 1) {
      cut = c == 1 ? 0xffff0000u : 0u;
      cut2 = 0u;
      unit = c < 2 ? 1.f : 0.f;
    } else {
      cut = c >= 1 ? 0xffff0000u : 0u;
      cut2 = c >= 2 ? 0xffff0000u : 0u;
      unit = c < 3 ? 1.f : 0.f;
    }
    l_run = 0.f;
    m_run = kNegInf;
    m_ref = 0.f;
#pragma unroll
    for (int e = 0; e < EV; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // The part of the logits that a term of K gives with the queries' first TERMS terms, added to c.
  template <int TERMS>
  static __device__ __forceinline__ void products(const uint32_t (&k)[NJ][2][4], const bf16x8_t (&qop)[NQ][2], f32x4_t (&c)[NJ]) {
#pragma unroll
    for (int n = 0; n < TERMS; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const u32x4_t a = {k[j][e][0], k[j][e][1], k[j][e][2], k[j][e][3]};
          c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), qop[n][e], c[j], 0, 0, 0);
        }
  }

  // From a tile's products to the weights of this lane's four tokens, of which those below `left` exist: they are 4 i + g.
  __device__ __forceinline__ void softmax(const f32x4_t (&c)[NJ], float k_scale, int left, int g, bool second, float (&p)[4]) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (NJ == 1)
        x[i] = c[0][i];
      else
        x[i] = quad_perm_add<0xB1>(second ? c[i / 2][i % 2 * 2 + 1] : c[i / 2][i % 2 * 2]);
      x[i] *= k_scale;
      if (left < kTile) x[i] = 4 * i + g < left ? x[i] : kNegInf;
    }
    const float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0ull) {
      const float most = rows_max(mx);
      const float m_new = most > m_run ? most + kGrow : m_run;
      m_ref = m_new == kNegInf ? 0.f : m_new;  // (finite before the first logit: -inf - -inf is no number)
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_ref);
      l_run *= alpha;
#pragma unroll
      for (int e = 0; e < EV; ++e) acc[e] *= alpha;
      m_run = m_new;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(x[i] - m_ref);
    l_run += (p[0] + p[1]) + (p[2] + p[3]);
  }

  // The operand of PV: this class's term of the weights times V's scale (TURN 1: the third term, in class 0).
  template <int TURN>
  __device__ __forceinline__ s16x4_t weights(const float (&p)[4], float v_scale) const {
    uint32_t t[4];
    const float s = TURN == 0 || kTurns == 1 ? v_scale * unit : v_scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float w = p[i] * s;
      if constexpr (NQ == 1) {  // both rounded: half a step is added before the lower half goes
        w -= __uint_as_float((__float_as_uint(w) + 0x8000u) & cut);
        t[i] = __float_as_uint(w) + 0x8000u;
      } else if constexpr (TURN == 0) {
        w -= __uint_as_float(__float_as_uint(w) & cut);
        if constexpr (GW == 4) w -= __uint_as_float(__float_as_uint(w) & cut2);
        t[i] = __float_as_uint(w);
      } else {
        w -= __uint_as_float(__float_as_uint(w) & 0xffff0000u);
        w -= __uint_as_float(__float_as_uint(w) & 0xffff0000u);
        t[i] = __float_as_uint(w) & ~cut;  // (class 1 has had its term)
      }
    }
    const u32x2_t packed = {__builtin_amdgcn_perm(t[1], t[0], 0x07060302u), __builtin_amdgcn_perm(t[3], t[2], 0x07060302u)};
    return __builtin_bit_cast(s16x4_t, packed);
  }

  __device__ __forceinline__ void add(int e, uint32_t lo, uint32_t hi, const s16x4_t& w) {
    const u32x2_t a = {lo, hi};
    acc[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, a), w, acc[e], 0, 0, 0);
  }
  // Four tokens' e4m3 numbers: of each two words, elements 0 and 1, then 2 and 3, side by side.
  __device__ __forceinline__ void accumulate(const VLoad (&v)[4], const s16x4_t (&w)[kTurns]) {
#pragma unroll
    for (int d = 0; d < EV / 4; ++d) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t sel = half ? 0x07030602u : 0x05010400u;
        const uint32_t lo = __builtin_amdgcn_perm(v[1][d], v[0][d], sel), hi = __builtin_amdgcn_perm(v[3][d], v[2][d], sel);
#pragma unroll
        for (int n = 0; n < kTurns; ++n) {
          add(4 * d + 2 * half, widen2<false>(lo), widen2<false>(hi), w[n]);
          add(4 * d + 2 * half + 1, widen2<true>(lo), widen2<true>(hi), w[n]);
        }
      }
    }
  }
  // The same of bfloat16 words.
  __device__ __forceinline__ void accumulate_words(const uint32_t (&v)[4][EV / 2], const s16x4_t (&w)[kTurns]) {
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
      const uint32_t lo = __builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], sel), hi = __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], sel);
#pragma unroll
      for (int n = 0; n < kTurns; ++n) add(e, lo, hi, w[n]);
    }
  }
};

template <typename T, int D, int GW, int WAVES, int DEPTH, bool SHARED, bool TAGGED>
__global__ __launch_bounds__(WAVES * kWave, 2) void quant_decode_kernel(
    const int32_t* seq_lens, const int32_t* block_table, const void* k_pool, const void* v_pool, const float* scales,
    const int num_kv_heads, const int max_blocks, const uint32_t inv_heads, const uint32_t shape, const QuantParams p) {
  using TL = Tile<T, D, GW>;
  using VLoad = typename TL::VLoad;
  using TM = Terms<T>;
  constexpr int NJ = TL::NJ, EV = TL::EV, NQ = TL::NQ;
  constexpr int GH = 16 / GW;  // heads computed; g_real of them exist
  // The tail without the first 8-bit tiles on their way: their registers then leave two workgroups of eight waves a place on a compute unit (320 rows x 1024
  // of fp32, D = 128, 21.2 us for 24.5, 288 of three tokens 4.8 / 6.9, 1024 x 2048 94 / 102; 64 rows x 1024 in four, which do not need it, 9.2 / 8.8).
  constexpr bool kTailAlone = NQ == 3 && D == 128;

  __shared__ WaveStates<WAVES, GH, D> sm;

  const int log2_block = shape_log2_block(shape), g_real = shape_group(shape), splits = shape_splits(shape);
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int g = lane >> 4, m = lane & 15, c = m % GW, h = m / GW;
  const Place at = decode_place(shape, num_kv_heads, inv_heads);
  const int row = at.row, split = at.split, s = at.seq, hk = at.head;
  const int32_t* bt = block_table + (int64_t)(SHARED ? s : row) * max_blocks;
  const int stride = splits * WAVES, first = split * WAVES + wave;
  const int tiles_log2 = log2_block - ilog2(kTile), in_page = (1 << tiles_log2) - 1;

  // (an unused entry, -1, is replaced by page 0: its tokens are behind the row's end and masked, so any address inside the pool will do.  A page
  // that is missing in front of the end, which an append without a spare page leaves behind, is the caller's: what is read there is page 0.)
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
  tl.begin(c);
  const int row_bytes = SHARED ? D * num_kv_heads : D;  // between consecutive tokens of this head
  const int k_tok = D == 64 ? 4 * (m & 3) + (m >> 2) : 4 * (m >> 1 & 1) + (m >> 2);  // of load 0; load j is 8 further
  const int k_elem = (D == 64 ? 0 : 64 * (m & 1)) + 16 * g;
  const int k_off = k_tok * row_bytes + (SHARED ? hk * D : 0) + k_elem;
  const int v_off = g * row_bytes + (SHARED ? hk * D : 0) + EV * m;

  // (a length that the table does not hold is a caller error: the table row is the end)
  const int len = len_raw < 0 ? 0 : (len_raw >> log2_block) < max_blocks ? len_raw : max_blocks << log2_block;
  const int full = len >> log2_block << log2_block;  // tokens in 8 bits
  const int ntiles = full >> ilog2(kTile), tail_tiles = (len - full + kTile - 1) >> ilog2(kTile);
  const int tail0 = stride - 1 - first;

  if (first < ntiles || tail0 < tail_tiles) {
    const auto base_of = [&](int tile, int ph) { return (((int64_t)ph << log2_block) + ((tile & in_page) * kTile)) * row_bytes; };
    // Loads are issued unconditionally, past the end all lanes fetch the pool's first bytes: the order of outstanding loads is known at
    // compile time, so that waiting for the oldest leaves the younger ones in flight.
    const auto issue_k = [&](u32x4_t(&buf)[NJ], int64_t base, int off, int step) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        buf[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(static_cast<const char*>(k_pool) + base + off + j * step));
    };
    const auto issue_v = [&](VLoad(&buf)[4], int64_t base, int off, int step) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        buf[i] = __builtin_nontemporal_load(reinterpret_cast<const VLoad*>(static_cast<const char*>(v_pool) + base + off + i * step));
    };
    const auto scales_of = [&](int ph) {
      const float* at = scales + ((int64_t)ph * (SHARED ? num_kv_heads : 1) + (SHARED ? hk : 0)) * 2;
      return make_float2(at[0], at[1]);
    };
    u32x4_t kb[DEPTH][NJ];
    VLoad vb[DEPTH][4];
    float2 sc[DEPTH];
    const auto begin_loads = [&] {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const bool more = first + d * stride < ntiles;
        const int64_t there = base_of(first + d * stride, phys[d]), base = more ? there : 0;
        issue_k(kb[d], base, more ? k_off : 0, more ? 8 * row_bytes : 0);
        issue_v(vb[d], base, more ? v_off : 0, more ? 4 * row_bytes : 0);
        sc[d] = scales_of(more ? phys[d] : 0);
      }
    };
    if constexpr (!kTailAlone) begin_loads();
    // queries: what faces a lane's elements of K, of the column's head and part
    bf16x8_t qop[NQ][2];
    const int64_t q_head = (int64_t)s * num_kv_heads * g_real + hk * g_real + (h < g_real ? h : 0);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t raw[4 * TM::kWords], t[4];
      TM::template load<8>(p.q, q_head * D + (D == 64 ? 0 : 64 * (c & 1)) + 16 * g + 8 * e, raw);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        TM::template take<8>(raw, t);
        const u32x4_t w = {t[0], t[1], t[2], t[3]}, zero = {0u, 0u, 0u, 0u};
        qop[n][e] = __builtin_bit_cast(bf16x8_t, h < g_real ? w : zero);
      }
    }

    // [S][Hk][B][D] in either layout
    for (int tail = tail0; tail < tail_tiles; tail += stride) {
      const int left = len - full - tail * kTile;
      const int64_t token0 = ((int64_t)row << log2_block) + tail * kTile;
      uint32_t kt[NJ][2][4 * TM::kWords], vt[4][EV / 2 * TM::kWords];
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) TM::template load<8>(p.k_tail, (token0 + k_tok + 8 * j) * D + k_elem + 8 * e, kt[j][e]);
#pragma unroll
      for (int i = 0; i < 4; ++i) TM::template load<EV>(p.v_tail, (token0 + 4 * i + g) * D + EV * m, vt[i]);
      f32x4_t prod[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) prod[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      float w[4];
      s16x4_t pop[TL::kTurns];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        uint32_t k[NJ][2][4];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) TM::template take<8>(kt[j][e], k[j][e]);
        if (n < 2)
          TL::template products<NQ>(k, qop, prod);
        else
          TL::template products<(NQ > 2 ? 2 : 1)>(k, qop, prod);
      }
      tl.softmax(prod, p.scale_log2e, left < kTile ? left : kTile, g, (c & 1) != 0, w);
      pop[0] = tl.template weights<0>(w, 1.f);
      if constexpr (TL::kTurns == 2) pop[1] = tl.template weights<1>(w, 1.f);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        uint32_t v[4][EV / 2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          TM::template take<EV>(vt[i], v[i]);
#pragma unroll
          for (int j = 0; j < EV / 2; ++j) v[i][j] = 4 * i + g < left ? v[i][j] : 0u;  // (what is no token may be anything)
        }
        tl.accumulate_words(v, pop);
      }
      if (WAVES * kTile >= kMostBlock) break;  // (a page's tiles: no wave has two)
    }

    if constexpr (kTailAlone) begin_loads();
    int ph_next = phys[DEPTH];
    for (int tile0 = first; tile0 < ntiles; tile0 += DEPTH * stride) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int tile = tile0 + d * stride;  // past the end (an odd last one): every token is masked
        const int left = DEPTH == 1 || tile < ntiles ? kTile : 0;
        uint32_t k[NJ][2][4];
        f32x4_t prod[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          prod[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w0 = kb[d][j][2 * e], w1 = kb[d][j][2 * e + 1];
            k[j][e][0] = widen2<false>(w0), k[j][e][1] = widen2<true>(w0), k[j][e][2] = widen2<false>(w1), k[j][e][3] = widen2<true>(w1);
          }
        }
        TL::template products<NQ>(k, qop, prod);
        const int ahead = tile + DEPTH * stride;
        const bool more = ahead < ntiles;
        const int64_t there = base_of(ahead, ph_next), base = more ? there : 0;
        const float2 now = sc[d];
        sc[d] = scales_of(more ? ph_next : 0);
        ph_next = lookup(ahead + stride);
        issue_k(kb[d], base, more ? k_off : 0, more ? 8 * row_bytes : 0);
        float w[4];
        s16x4_t pop[TL::kTurns];
        tl.softmax(prod, now.x * p.scale_log2e, left, g, (c & 1) != 0, w);
        const float v_scale = DEPTH == 1 || left ? now.y : 0.f;
        pop[0] = tl.template weights<0>(w, v_scale);
        if constexpr (TL::kTurns == 2) pop[1] = tl.template weights<1>(w, v_scale);
        if constexpr (DEPTH > 1) {
          if (!left) {
#pragma unroll
            for (int i = 0; i < 4; ++i) vb[d][i] = VLoad(0u);
          }
        }
        tl.accumulate(vb[d], pop);
        issue_v(vb[d], base, more ? v_off : 0, more ? 4 * row_bytes : 0);
      }
    }
    // (the placeholder loads behind a wave's last tiles: their registers are in use until they are back)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : : "v"(kb[d][j]));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < EV / 4; ++e) asm volatile("" : : "v"(vb[d][i][e]));
    }
  }

  // ---- merge: classes, lane groups, then the waves through LDS -------------------------------
  // C[slice][column] of element e: lane (g, m) has slices 4 g .. 4 g + 3 of its head; each class stores 4 / GW of them.
  {
    const float l = rows_sum(tl.l_run);
    if (g == 0 && c == 0) sm.ml[wave][h] = make_float2(tl.m_run, l);
    float o[4 / GW][EV];
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      float a[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) a[r] = class_sum<GW>(tl.acc[e][r]);
      if constexpr (GW == 4) {
        const float lo = (c & 1) ? a[1] : a[0], hi = (c & 1) ? a[3] : a[2];
        o[0][e] = (c & 2) ? hi : lo;
      } else {
        o[0][e] = c ? a[2] : a[0];
        o[1][e] = c ? a[3] : a[1];
      }
    }
#pragma unroll
    for (int r = 0; r < 4 / GW; ++r) {
      float4* dst = reinterpret_cast<float4*>(&sm.acc[wave][h][(4 * g + c * (4 / GW) + r) * EV]);
#pragma unroll
      for (int e = 0; e < EV / 4; ++e) dst[e] = make_float4(o[r][4 * e], o[r][4 * e + 1], o[r][4 * e + 2], o[r][4 * e + 3]);
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

template <typename T, int D, int GW, int WAVES, int DEPTH>
hipError_t launch_one(const QuantDecodeArgs& a, hipStream_t stream) {
  PlaceGrid grid;
  if (!place_grid(a.num_seqs, a.num_kv_heads, a.splits, true, &grid)) return hipErrorInvalidValue;
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const uint32_t shape = (uint32_t)log2_block | (uint32_t)(a.num_q_heads / a.num_kv_heads) << 3 | (grid.xcd ? kShapeXcd : 0u) |
                         (grid.linear ? kShapeLinear : 0u) | (uint32_t)a.splits << 9;
  QuantKernel kernel = a.shared ? quant_decode_kernel<T, D, GW, WAVES, DEPTH, true, false> : quant_decode_kernel<T, D, GW, WAVES, DEPTH, false, false>;
  if (a.tagged) {
    if constexpr (one_part_a_wave<16 / GW, D, WAVES>)
      kernel = a.shared ? quant_decode_kernel<T, D, GW, WAVES, DEPTH, true, true> : quant_decode_kernel<T, D, GW, WAVES, DEPTH, false, true>;
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
  if (a.waves == 4) return wide ? launch_one<T, D, 2, 4, 1>(a, stream) : launch_one<T, D, 4, 4, 1>(a, stream);
  if constexpr (D == 64) {
    if (a.depth == 2) return wide ? launch_one<T, D, 2, 8, 2>(a, stream) : launch_one<T, D, 4, 8, 2>(a, stream);
  }
  return wide ? launch_one<T, D, 2, 8, 1>(a, stream) : launch_one<T, D, 4, 8, 1>(a, stream);
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
