// Attention of several query rows that share the K and V of a row of the cache (Eq. 1), on the matrix cores: trees of drafted
// tokens (up to 64 queries per sequence and head), and one query a sequence with the weight that each page got.
//
// A row, (sequence, KV head), has R = drafts x G query rows (r = draft * G + head of the group) that read the same K and V: the
// L cached tokens, and behind them the drafts' own keys, of which each query row sees those that its draft's mask names.  A
// workgroup owns 16 * NQ query rows and one split of the tokens; its four waves take STEP tokens at a time, all query rows
// each, so that every element of K and V goes from memory to the registers of one wave and from there into the products.
// Tokens are dealt out in rounds of 128 (the drafts are a round of their own behind the cache's), round t to split t % splits, so
// that a page lies in one split and a wave's first step does not depend on the row's length.
//
// With lane l = 16*g + n:
//   QK (A = K, B = Q): C[m][n] = <k_m, q_n>, tokens in rows, queries in columns.  Lane l loads 16 bytes of token n (as row m)
//   at chunk 4*j + g; the contraction runs over the chunks, and Q is loaded by the same map.  Lane l is left with the logits of
//   tokens 4*g + r of query n, r < 4.
//   PV (A = V transposed, B = P): out^T[d][n] = sum_t V[t][d] P[t][n].  The logits' registers are the B operand as they lie
//   (contraction index: the tokens 4*g + r of the step's 16-token parts), and row m of A is d = m*E + e in product e, E = D/16
//   (fp32: d = 64*(e/4) + 4*m + e%4): lane l loads those of row n of its tokens 4*g + r, whole runs of a token for 16 lanes.
//   bfloat16 products contract 32 tokens (two parts), fp32 ones four, one for each r.
//
// bfloat16: a probability goes into the product as two bfloat16 terms, within 2^-17 of it (terms_of): one product more of each, and a
// rounding of the probabilities that is small beside that of the output.
//
// Softmax: online, base 2, a reference per query row and wave that is set kGrow above the largest logit and moves only when one
// exceeds it, so that rescaling is rare.  What no row attends to (a token behind the row's end, a draft behind the sequence's
// last) is taken out of V as well, where anything may lie.  A query row that attends to nothing gives zeros.
//
// Page weights (WEIGHTS): the sum of a part's probabilities is kept in LDS with the reference it is relative to (a store to memory
// there would turn every wait for a load into a full one), and when the row's sums are known a page's weight is that of its parts.
// With several splits each writes its pages' sums, and the launch that merges the splits makes the weights.
//
// What bounds it is reading K and V: eight heads of D = 128, 32 sequences, 8 drafts x 4 heads over 1024 to 2048 tokens 42.5 us (4.8 TB/s; the
// last workgroups have the longest rows to themselves), one query with weights over 2033 to 2048 tokens 45 (5.9 TB/s).  Few rows are bound by
// the chain of a launch (length, page, K, products, merge): one sequence of 1000 tokens, 4 x 4 heads of D = 64, 6 us and 2.4 for the merge of
// its splits: 0.8 until the length is there, as much again for the first K, 0.6 for the step, 0.9 each for the drafts' and the end.  fp32 of
// D = 128 takes 1.7 us a step (16 tokens a wave).  Not faster, over 20 shapes: eight waves (42.5 / 44 and 10.1 / 10.6 us), two steps of a
// wave on their way (8.6 / 9.4 for the 1000 tokens, 45 / 46 for the weights: what a wave asks for behind its last step costs more than the
// wait saves), no loads behind the last step (8.6 / 8.2, but 44 / 46.5 for the batch), fp32 products of four columns (18.5 / 18.6).
#include "pe_rows_device.h"

namespace pe {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
static_assert(kThreads == kRowsThreads && kWaves == kMergeRows, "what the host counts with");

// Row geometry: elements of a 16-byte K chunk, chunks a lane loads of a token, elements of V a lane loads of a token.
template <typename T, int D>
struct Geo {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kStep = kBf16 ? 32 : 16;  // tokens of a step
  static constexpr int kParts = kStep / 16;
  static constexpr int kPerRound = kRoundTokens / (kWaves * kStep);  // steps of a wave in a round
  static constexpr int kElems = 16 / (int)sizeof(T);
  static constexpr int kChunks = D / kElems / 4;  // K: chunks a lane loads
  static constexpr int E = D / 16;                // V: elements a lane loads of a token
  static constexpr int kVDwords = E * (int)sizeof(T) / 4;
  // The element of V that a lane's element e is, for lane n (row n of the product): 16 bytes a lane (D = 64, bfloat16: 8), so that
  // 16 neighbouring lanes read 256 consecutive bytes.
  static __device__ __forceinline__ int element_of(int n, int e) { return kBf16 ? n * E + e : e / 4 * 64 + n * 4 + e % 4; }
};

// The weight of a page, from what earlier calls left and what this one adds.
__device__ __forceinline__ void put_weight(const RowsParams& p, int64_t at, float got) {
  float before = 0.f;
  if (p.weights_in != nullptr) {
    const float w = p.weights_in[at];
    before = fabsf(w) < __builtin_inff() ? w : 0.f;  // (what is no number counts as nothing: a page's first time)
  }
  p.weights_out[at] = fmaf(before, p.decay, got);
}

template <typename T, int D, int NQ, bool WEIGHTS>
__global__ __launch_bounds__(kThreads, 2) void paged_rows_kernel(const RowsParams p) {
  using GE = Geo<T, D>;
  constexpr int STEP = GE::kStep, PARTS = GE::kParts, CH = GE::kChunks, E = GE::E, VD = GE::kVDwords, PER = GE::kPerRound;
  constexpr int ROWS = 16 * NQ;
  static_assert(!WEIGHTS || NQ == 1, "one query a sequence");
  __shared__ __attribute__((aligned(16))) float sm_acc[kWaves][16][D + 4];
  __shared__ float2 sm_ml[kWaves][16];
  extern __shared__ float2 sm_parts[];  // WEIGHTS: [part of the split][G] (sum, reference)

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int g = lane >> 4, n = lane & 15;
  const int log2_block = shape_log2_block(p.shape), group = shape_group(p.shape), splits = shape_splits(p.shape);
  const int tiles = WEIGHTS ? 1 : p.tiles;
  const Place at = place_at(blockIdx.x, blockIdx.y, (p.shape & kShapeXcd) != 0, (p.shape & kShapeLinear) != 0, splits * tiles, p.num_kv_heads,
                            p.inv_heads);
  const int s = at.seq, hk = at.head;
  const int split = WEIGHTS || tiles == 1 ? at.split : at.split / tiles, tile = at.split - split * tiles;
  const bool shared = p.max_blocks < 0;
  const int max_blocks = shared ? -p.max_blocks : p.max_blocks;
  // (read only while the launch runs: scalar loads, also behind a barrier or a store)
  const auto* table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
      reinterpret_cast<uintptr_t>(p.block_table + (int64_t)(shared ? s : at.row) * max_blocks));

  // Step k of this wave: its round and the first token in it.
  const auto round_of = [&](int k) { return split + k / PER * splits; };
  const auto inside = [&](int k) { return k % PER * (kWaves * STEP) + wave * STEP; };
  // Pages of its parts (scalar loads; clamped to the table row, nothing here depends on the row's length).
  const auto lookup = [&](int k, int (&ids)[PARTS]) __attribute__((always_inline)) {
    const int64_t tok = (int64_t)round_of(k) * kRoundTokens + inside(k);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const int64_t j = (tok + part * 16) >> log2_block;
      ids[part] = table[j < max_blocks ? (int)j : max_blocks - 1];
    }
  };
  int ids[PARTS], ids_next[PARTS];
  lookup(0, ids);
  lookup(1, ids_next);
  const int len = length_of(p, s, max_blocks, log2_block);
  const int drafts = WEIGHTS ? 1 : drafts_of(p, s);
  const int rows = drafts * group, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int cached = len / kRoundTokens + (len % kRoundTokens != 0), rounds = cached + (WEIGHTS ? 0 : 1);

  uint4 kb[PARTS][CH];
  uint32_t vb[PARTS][4][VD];
  const uint32_t token_bytes = (uint32_t)(shared ? p.num_kv_heads : 1) * (D * (uint32_t)sizeof(T));   // of a page
  const uint32_t draft_bytes = (uint32_t)p.num_kv_heads * (D * (uint32_t)sizeof(T));
  // (the drafts' places as distances from the pools': a choice between two arguments would load the chosen one every time)
  const int64_t k_far = WEIGHTS ? 0 : static_cast<const char*>(p.k_draft) - static_cast<const char*>(p.k_pool);
  const int64_t v_far = WEIGHTS ? 0 : static_cast<const char*>(p.v_draft) - static_cast<const char*>(p.v_pool);
  const auto load = [&](int k, const int (&id)[PARTS], bool keys) __attribute__((always_inline)) {
    const int round = round_of(k);
    const bool pool = WEIGHTS || round < cached;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      int tok = inside(k) + part * 16;   // of the round; what is no token reads one that is
      uint32_t stride = token_bytes, last = 15u;
      const bool in = round < cached;  // (a part behind the row's end lies in its table row, or is replaced)
      const int page = id[part] < 0 || !in ? 0 : id[part];
      const int slot = (int)(((int64_t)round * kRoundTokens + tok) & ((1 << log2_block) - 1));
      int64_t from = (((int64_t)page << log2_block) + slot) * token_bytes + (shared ? hk * (D * (int)sizeof(T)) : 0);
      if (!pool) {
        const int end = round == cached ? drafts : 1;
        tok = tok < end ? tok : 0;
        last = (uint32_t)(end - 1 - tok < 15 ? end - 1 - tok : 15);
        stride = draft_bytes;
        from = ((int64_t)s * p.drafts + tok) * draft_bytes + hk * (D * (int)sizeof(T)) + (keys ? k_far : v_far);
      }
      const char* base = static_cast<const char*>(keys ? p.k_pool : p.v_pool) + from;
      if (keys) {
        const uint32_t off = ((uint32_t)n < last ? (uint32_t)n : last) * stride + (uint32_t)g * 16u;
#pragma unroll
        for (int j = 0; j < CH; ++j) kb[part][j] = load_vec(base + off, j * 4);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t t = (uint32_t)(4 * g + r);
          const uint32_t off = (t < last ? t : last) * stride + (uint32_t)n * (VD >= 4 ? 16u : 8u);
          if constexpr (VD >= 4) {
#pragma unroll
            for (int w = 0; w < VD; w += 4) {
              const uint4 v = load_vec_stream(base + off, w * 4);
              vb[part][r][w] = v.x, vb[part][r][w + 1] = v.y, vb[part][r][w + 2] = v.z, vb[part][r][w + 3] = v.w;
            }
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(base + off);
            vb[part][r][0] = v.x, vb[part][r][1] = v.y;
          }
        }
      }
    }
  };

  // ---- first loads: K, the queries, V ------------------------------------------------------------------------------------
  const int num_q_heads = p.num_kv_heads * group;
  uint4 q[NQ][CH];
  uint64_t sees[NQ];  // drafts that the lane's query row attends to
  load(0, ids, true);
  // (In this order: what is waited for first in the loop, K, has V behind it there, and the queries must not lie in between.)
  __builtin_amdgcn_sched_barrier(0);
  const uint64_t real = drafts >= 64 ? ~0ull : (1ull << drafts) - 1;
#pragma unroll
  for (int a = 0; a < NQ; ++a) {
    const int r = row0 + 16 * a + n;  // (behind the last one: the first one again, and written nowhere)
    int draft = 0, h = r < rows ? r : 0;
    if constexpr (!WEIGHTS) {
      draft = h / group;
      h -= draft * group;
    }
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) +
                                                       (((int64_t)s * (WEIGHTS ? 1 : p.drafts) + draft) * num_q_heads + hk * group + h) * D);
#pragma unroll
    for (int j = 0; j < CH; ++j) q[a][j] = from[4 * j + g];
    sees[a] = WEIGHTS ? 0ull : p.mask[(int64_t)s * p.drafts + draft] & real;
  }
  __builtin_amdgcn_sched_barrier(0);
  load(0, ids, false);
  __builtin_amdgcn_sched_barrier(0);

  f32x4_t acc[NQ][E];
  float m_run[NQ], m_ref[NQ], l_run[NQ];
#pragma unroll
  for (int a = 0; a < NQ; ++a) {
    m_run[a] = kNegInf;
    m_ref[a] = 0.f;
    l_run[a] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[a][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  for (int k = 0; round_of(k) < rounds; ++k) {
    const int round = round_of(k);
    const bool pool = WEIGHTS || round < cached;
    const int tok0 = inside(k), end = pool ? len - round * kRoundTokens : drafts;  // of the round
    f32x4_t x[NQ][PARTS];
#pragma unroll
    for (int a = 0; a < NQ; ++a)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) x[a][part] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < CH; ++j)  // (neighbouring products add to different sums)
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
#pragma unroll
        for (int a = 0; a < NQ; ++a) {
          f32x4_t& c = x[a][part];
          if constexpr (GE::kBf16) {
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kb[part][j]), __builtin_bit_cast(bf16x8_t, q[a][j]),
                                                        c, 0, 0, 0);
          } else {
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kb[part][j].x), __uint_as_float(q[a][j].x), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kb[part][j].y), __uint_as_float(q[a][j].y), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kb[part][j].z), __uint_as_float(q[a][j].z), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kb[part][j].w), __uint_as_float(q[a][j].w), c, 0, 0, 0);
          }
        }
#pragma unroll
    for (int a = 0; a < NQ; ++a)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) x[a][part] *= p.scale_log2e;
    load(k + 1, ids_next, true);
    if (!pool || tok0 + STEP > end) {
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = tok0 + part * 16 + 4 * g + r;
          if (t >= end) {
#pragma unroll
            for (int w = 0; w < VD; ++w) vb[part][r][w] = 0u;
          }
#pragma unroll
          for (int a = 0; a < NQ; ++a) {
            const bool in = pool ? t < end : (t < kMostDrafts && ((sees[a] >> (t & 63)) & 1u) != 0);
            if (!in) x[a][part][r] = kNegInf;
          }
        }
    }
#pragma unroll
    for (int a = 0; a < NQ; ++a) {
      float mx = kNegInf;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) mx = fmaxf(mx, fmaxf(fmaxf(x[a][part][0], x[a][part][1]), fmaxf(x[a][part][2], x[a][part][3])));
      if (__builtin_amdgcn_ballot_w64(mx > m_run[a]) != 0ull) {
        mx = rows_max(mx);
        const float m_new = mx > m_run[a] ? mx + kGrow : m_run[a];
        const float ref = m_new == kNegInf ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run[a] - ref);
        l_run[a] *= alpha;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[a][e] *= alpha;
        m_run[a] = m_new;
        m_ref[a] = ref;
      }
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
#pragma unroll
        for (int r = 0; r < 4; ++r) x[a][part][r] = __builtin_amdgcn_exp2f(x[a][part][r] - m_ref[a]);
        const float sum = (x[a][part][0] + x[a][part][1]) + (x[a][part][2] + x[a][part][3]);
        l_run[a] += sum;
        if constexpr (WEIGHTS) {
          const float whole = rows_sum(sum);
          if (lane < group) sm_parts[(k / PER * (kRoundTokens / 16) + tok0 / 16 + part) * group + lane] = make_float2(whole, m_ref[a]);
        }
      }
    }
    if constexpr (GE::kBf16) {
      bf16x8_t hi[NQ], lo[NQ];
#pragma unroll
      for (int a = 0; a < NQ; ++a) {
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const Terms t = terms_of(x[a][w / 2][w % 2 * 2], x[a][w / 2][w % 2 * 2 + 1]);
          hw[w] = t.hi;
          lw[w] = t.lo;
        }
        hi[a] = __builtin_bit_cast(bf16x8_t, make_uint4(hw[0], hw[1], hw[2], hw[3]));
        lo[a] = __builtin_bit_cast(bf16x8_t, make_uint4(lw[0], lw[1], lw[2], lw[3]));
      }
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        bf16x8_t v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t sel = i != 0 ? 0x07060302u : 0x05040100u;
          v[i] = __builtin_bit_cast(bf16x8_t, make_uint4(__builtin_amdgcn_perm(vb[0][1][e >> 1], vb[0][0][e >> 1], sel),
                                                         __builtin_amdgcn_perm(vb[0][3][e >> 1], vb[0][2][e >> 1], sel),
                                                         __builtin_amdgcn_perm(vb[PARTS - 1][1][e >> 1], vb[PARTS - 1][0][e >> 1], sel),
                                                         __builtin_amdgcn_perm(vb[PARTS - 1][3][e >> 1], vb[PARTS - 1][2][e >> 1], sel)));
        }
#pragma unroll
        for (int term = 0; term < 2; ++term)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int a = 0; a < NQ; ++a)
              acc[a][e + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[i], term == 0 ? hi[a] : lo[a], acc[a][e + i], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int a = 0; a < NQ; ++a)
            acc[a][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vb[0][r][e]), x[a][0][r], acc[a][e], 0, 0, 0);
    }
    load(k + 1, ids_next, false);
    lookup(k + 2, ids_next);
  }

  // ---- the waves' states, 16 query rows at a time ---------------------------------------------------------------------
#pragma unroll
  for (int a = 0; a < NQ; ++a) {
    const float l = rows_sum(l_run[a]);
    if (g == 0) sm_ml[wave][n] = make_float2(m_run[a], l);
    // lane (g, n) has rows m = 4*g + r of C: elements element_of(m, e) of query n
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(&sm_acc[wave][n][GE::element_of(4 * g + r, e)]) =
            make_float4(acc[a][e][r], acc[a][e + 1][r], acc[a][e + 2][r], acc[a][e + 3][r]);
    }
    __syncthreads();
    for (int idx = (int)threadIdx.x; idx < 16 * (D / 2); idx += kThreads) {
      const int i = idx / (D / 2), d = idx % (D / 2) * 2, r = row0 + 16 * a + i;
      if (r >= rows) continue;
      float m = kNegInf, lsum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sm_ml[w][i].x);
      const float ms = m == kNegInf ? 0.f : m;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_ml[w][i].x - ms);
        lsum = fmaf(sm_ml[w][i].y, f, lsum);
        o0 = fmaf(sm_acc[w][i][d], f, o0);
        o1 = fmaf(sm_acc[w][i][d + 1], f, o1);
      }
      if (splits == 1) {
        const int draft = WEIGHTS ? 0 : r / group, h = r - draft * group;
        const int64_t head = ((int64_t)s * (WEIGHTS ? 1 : p.drafts) + draft) * num_q_heads + hk * group + h;
        store_pair<T>(p.out, (head * D + d) / 2, lsum > 0.f ? o0 / lsum : 0.f, lsum > 0.f ? o1 / lsum : 0.f);
      } else {
        const int most = (WEIGHTS ? 1 : p.drafts) * group;
        float* record = p.partials + ((((int64_t)hk * p.num_seqs + s) * splits + split) * most + r) * (D + 2);
        *reinterpret_cast<float2*>(record + d) = make_float2(o0, o1);
        if (d == 0) *reinterpret_cast<float2*>(record + D) = make_float2(m, lsum);
      }
    }
    if (a + 1 < NQ) __syncthreads();
  }

  if constexpr (WEIGHTS) {
    // page t of the split's: of its local round t / (pages of a round)
    const int per_round = kRoundTokens >> log2_block, parts = 1 << (log2_block - 4);
    const int pages = (int)(((int64_t)len + (1 << log2_block) - 1) >> log2_block);
    const int my_rounds = cached > split ? (cached - split + splits - 1) / splits : 0;
    for (int t = (int)threadIdx.x; t < my_rounds * per_round; t += kThreads) {
      const int local = t / per_round, j = (split + local * splits) * per_round + t % per_round;
      if (j >= pages) continue;
      const int left = (len - (j << log2_block) + 15) / 16, real_parts = left < parts ? left : parts;
      float got = 0.f;
      for (int h = 0; h < group; ++h) {
        float m = kNegInf, lsum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sm_ml[w][h].x);
        const float ms = m == kNegInf ? 0.f : m;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) lsum = fmaf(sm_ml[w][h].y, __builtin_amdgcn_exp2f(sm_ml[w][h].x - ms), lsum);
        float sum = 0.f;
        for (int i = 0; i < real_parts; ++i) {
          const float2 part = sm_parts[(t * parts + i) * group + h];
          sum = fmaf(part.x, __builtin_amdgcn_exp2f(part.y - ms), sum);
        }
        if (splits > 1)
          p.page_sums[((int64_t)at.row * max_blocks + j) * group + h] = sum;
        else
          got += sum / lsum;
      }
      if (splits == 1) put_weight(p, (int64_t)at.row * max_blocks + j, got);
    }
    if (splits == 1)
      for (int j = pages + (int)threadIdx.x; j < max_blocks; j += kThreads) p.weights_out[(int64_t)at.row * max_blocks + j] = __builtin_inff();
  }
}

// The splits of a query row, one wave each, added in their order: records from number `first` on.
template <typename T, int D>
__device__ __forceinline__ void merge_row(const RowsParams& p, int64_t first, int r, int most, int splits, int64_t head, int lane) {
  constexpr int E = D / kWave;
  const float* base = p.partials + (first * most + r) * (D + 2);
  float o[E];
  merge_splits<E>(splits, o, [&](int split, float2& ml, float (&v)[E]) {
    const float* record = base + (int64_t)split * most * (D + 2);
    ml = *reinterpret_cast<const float2*>(record + D);
    if constexpr (E == 2) {
      const float2 pair = *reinterpret_cast<const float2*>(record + lane * 2);
      v[0] = pair.x, v[1] = pair.y;
    } else {
      v[0] = record[lane];
    }
  });
  const int64_t to = head * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (sizeof(T) == 4)
      static_cast<float*>(p.out)[to + e] = o[e];
    else
      static_cast<uint16_t*>(p.out)[to + e] = f32_to_bf16(o[e]);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rows_merge_kernel(const RowsParams p) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int group = shape_group(p.shape), most = p.drafts * group, tiles = (most + kWaves - 1) / kWaves;
  const int row = (int)(blockIdx.x / (uint32_t)tiles), r = ((int)blockIdx.x - row * tiles) * kWaves + wave;
  const int s = row / p.num_kv_heads, hk = row - s * p.num_kv_heads;
  if (r >= drafts_of(p, s) * group) return;
  const int draft = r / group, h = r - draft * group, lane = lane_id();
  int splits = shape_splits(p.shape), first = s * splits;
  const int64_t head = (int64_t)hk * p.num_seqs * splits;
  if (p.shares != nullptr) first = (int)p.shares[2 * s], splits = (int)p.shares[2 * s + 1];
  merge_row<T, D>(p, head + first, r, most, splits, ((int64_t)s * p.drafts + draft) * (p.num_kv_heads * group) + hk * group + h, lane);
}

// The splits of a row and the weights of its pages, one workgroup a row.  A head's (m, l) of all splits are read at once, a split a lane, and
// a thread's first page while they are.
template <int M = 1>
__device__ __forceinline__ float wave_max(float v) {
  if constexpr (M == 16)
    return rows_max(v);
  else
    return wave_max<M * 2>(fmaxf(v, lane_xor_f32<M>(v)));
}
template <int M = 1>
__device__ __forceinline__ float wave_sum(float v) {
  if constexpr (M == 16)
    return rows_sum(v);
  else
    return wave_sum<M * 2>(v + lane_xor_f32<M>(v));
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void weights_merge_kernel(const RowsParams p) {
  __shared__ float factor[256][8];  // of a split and head: what turns its pages' sums into weights
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int group = shape_group(p.shape), splits = shape_splits(p.shape), log2_block = shape_log2_block(p.shape);
  const int row = (int)blockIdx.x, s = row / p.num_kv_heads;
  const int64_t first = ((int64_t)(row - s * p.num_kv_heads) * p.num_seqs + s) * splits;
  const bool shared = p.max_blocks < 0;
  const int max_blocks = shared ? -p.max_blocks : p.max_blocks;
  const int len = length_of(p, s, max_blocks, log2_block);
  const int pages = (int)(((int64_t)len + (1 << log2_block) - 1) >> log2_block);
  const int64_t row_at = (int64_t)row * max_blocks;
  const auto sums_of = [&](int j, float (&sums)[8]) {
#pragma unroll
    for (int h = 0; h < 8; ++h) sums[h] = h < group && j < pages ? p.page_sums[(row_at + j) * group + h] : 0.f;
  };
  float sums[8];
  sums_of((int)threadIdx.x, sums);
  for (int h = wave; h < group; h += kWaves) {
    const float* ml = p.partials + (first * group + h) * (D + 2) + D;
    const int64_t stride = (int64_t)group * (D + 2);
    float2 of[4];
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int split = i * kWave + lane;
      of[i] = split < splits ? *reinterpret_cast<const float2*>(ml + split * stride) : make_float2(kNegInf, 0.f);
      m = fmaxf(m, of[i].x);
    }
    merge_row<T, D>(p, first, h, group, splits, (int64_t)row * group + h, lane);
    m = wave_max(m);
    const float ms = m == kNegInf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i) l = fmaf(of[i].y, __builtin_amdgcn_exp2f(of[i].x - ms), l);
    l = wave_sum(l);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i * kWave + lane < splits) factor[i * kWave + lane][h] = l > 0.f ? __builtin_amdgcn_exp2f(of[i].x - ms) / l : 0.f;
  }
  __syncthreads();
  for (int j = (int)threadIdx.x; j < max_blocks; j += kThreads) {
    if (j != (int)threadIdx.x) sums_of(j, sums);
    if (j >= pages) {
      p.weights_out[row_at + j] = __builtin_inff();
      continue;
    }
    const int split = (int)((((int64_t)j << log2_block) / kRoundTokens) % splits);
    float got = 0.f;
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (h < group) got = fmaf(sums[h], factor[split][h], got);
    put_weight(p, row_at + j, got);
  }
}

template <typename T, int D, int NQ>
hipError_t launch_tiles(const RowsArgs& a, RowsParams p, hipStream_t stream) {
  dim3 blocks;
  const dim3 threads(kThreads);
  if (!rows_grid(a, 16 * NQ, &p, &blocks)) return hipErrorInvalidValue;
  if constexpr (NQ == 1) {
    if (a.weights_out != nullptr) {
      hipLaunchKernelGGL((paged_rows_kernel<T, D, 1, true>), blocks, threads, a.part_bytes, stream, p);
      if (a.splits > 1)
        hipLaunchKernelGGL((weights_merge_kernel<T, D>), dim3((unsigned)(a.num_seqs * a.num_kv_heads)), threads, 0, stream, p);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((paged_rows_kernel<T, D, NQ, false>), blocks, threads, 0, stream, p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_rows(const RowsArgs& a, const RowsParams& p, hipStream_t stream) {
  hipError_t rc = hipErrorInvalidValue;
  if (a.tile_rows == 16) rc = launch_tiles<T, D, 1>(a, p, stream);
  if (a.tile_rows == 32) rc = launch_tiles<T, D, 2>(a, p, stream);
  if constexpr (sizeof(T) == 2) {
    if (a.tile_rows == kWideRows) rc = launch_tree_wide(a, p, stream);
  }
  if (rc == hipSuccess && a.splits > 1 && a.weights_out == nullptr) {
    const int64_t merges = (int64_t)a.num_seqs * a.num_kv_heads * ((a.drafts * shape_group(p.shape) + kWaves - 1) / kWaves);
    hipLaunchKernelGGL((rows_merge_kernel<T, D>), dim3((unsigned)merges), dim3(kThreads), 0, stream, p);
    rc = hipGetLastError();
  }
  return rc;
}

}  // namespace

hipError_t launch_paged_rows(const RowsArgs& a, hipStream_t stream) {
  RowsParams p{};
  p.seq_lens = a.seq_lens, p.block_table = a.block_table;
  p.k_pool = a.k_pool, p.v_pool = a.v_pool;
  p.num_kv_heads = a.num_kv_heads, p.max_blocks = a.shared ? -a.max_blocks : a.max_blocks;
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  p.shape = (uint32_t)log2_block | (uint32_t)(a.num_q_heads / a.num_kv_heads) << 3 | (uint32_t)a.splits << 9;
  p.drafts = a.drafts, p.num_seqs = a.num_seqs, p.shares = a.shares;
  p.q = a.q;
  p.scale_log2e = a.scale * 1.4426950408889634f;
  p.decay = a.decay;
  p.draft_lens = a.draft_lens, p.mask = a.mask;
  p.k_draft = a.k_draft, p.v_draft = a.v_draft;
  p.out = a.out, p.partials = a.partials;
  p.weights_in = a.weights_in, p.weights_out = a.weights_out, p.page_sums = a.page_sums;
  if (a.is_bf16) return a.head_dim == 64 ? launch_rows<bf16_t, 64>(a, p, stream) : launch_rows<bf16_t, 128>(a, p, stream);
  return a.head_dim == 64 ? launch_rows<float, 64>(a, p, stream) : launch_rows<float, 128>(a, p, stream);
}

}  // namespace pe
