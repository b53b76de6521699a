// Attention of a tree of drafted tokens over a paged cache (Eq. 1 for up to 64 queries per sequence and head), on the matrix
// cores.
//
// A row, (sequence, KV head), has R = drafts x G query rows (r = draft * G + head of the group) that read the same K and V: the
// L cached tokens, and behind them the drafts' own keys, of which each query row sees those that its draft's mask names.  A
// workgroup owns 16 * NQ query rows and one split of the tokens; its four waves take steps of STEP tokens in turn, all query
// rows each, so that every element of K and V goes from memory to the registers of one wave and from there into the products.
//
// With lane l = 16*g + n:
//   QK (A = K, B = Q): C[m][n] = <k_m, q_n>, tokens in rows, queries in columns.  Lane l loads 16 bytes of token n (as row m)
//   at chunk 4*j + g; the contraction runs over the chunks, and Q is loaded by the same map.  Lane l is left with the logits of
//   tokens 4*g + r of query n, r < 4.
//   PV (A = V transposed, B = P): out^T[d][n] = sum_t V[t][d] P[t][n].  The logits' registers are the B operand as they lie
//   (contraction index: the tokens 4*g + r of the step's 16-token parts), and row m of A is d = m*E + e in product e, E = D/16:
//   lane l loads elements n*E .. n*E + E - 1 of its tokens 4*g + r, whole token rows for 16 neighbouring lanes.
//   bfloat16 products contract 32 tokens (two parts), fp32 ones four, one for each r.
//
// bfloat16: a probability goes into the product as two bfloat16 terms, p = hi + lo + less than 2^-16 p (hi the upper half of its
// bits, lo what they leave): one product more of each, and no rounding of the probabilities beside that of the output.
//
// Softmax: online, base 2, a reference per query row and wave that is set kGrow above the largest logit and moves only when one
// exceeds it, so that rescaling is rare.  What no row attends to (a token behind the row's end, a draft behind the sequence's
// last) is taken out of V as well, where anything may lie.  A query row that attends to nothing gives zeros.
#include "pe_decode_common.h"
#include "pe_tree.h"

namespace pe {
namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kGrow = 3.f;
constexpr int kWaves = 4;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

struct TreeParams {
  const void *q, *k_draft, *v_draft;
  const int32_t* draft_lens;  // or null: every sequence has all of them
  const uint64_t* mask;
  const void *k_pool, *v_pool;
  const int32_t *block_table, *seq_lens;
  void* out;
  float* partials;
  float scale_log2e;
  int num_kv_heads, group, drafts, max_blocks, log2_block;
  int splits, tiles;  // of a row: shares of the tokens, workgroups for its query rows
  uint32_t inv_heads;
  int xcd, linear;
};

// Row geometry: elements of a 16-byte K chunk, chunks a lane loads of a token, elements of V a lane loads of a token.
template <typename T, int D>
struct Geo {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kStep = kBf16 ? 32 : 16;  // tokens of a step
  static constexpr int kParts = kStep / 16;
  static constexpr int kElems = 16 / (int)sizeof(T);
  static constexpr int kChunks = D / kElems / 4;  // K: chunks a lane loads
  static constexpr int E = D / 16;                // V: elements a lane loads of a token
  static constexpr int kVDwords = E * (int)sizeof(T) / 4;
};

template <typename T, int D, int NQ>
__global__ __launch_bounds__(kWaves * kWave, NQ >= 4 ? 1 : 2) void tree_decode_kernel(const TreeParams p) {
  using GE = Geo<T, D>;
  constexpr int STEP = GE::kStep, PARTS = GE::kParts, CH = GE::kChunks, E = GE::E, VD = GE::kVDwords;
  constexpr int ROWS = 16 * NQ;
  __shared__ __attribute__((aligned(16))) float sm_acc[kWaves][16][D + 4];
  __shared__ float2 sm_ml[kWaves][16];

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int g = lane >> 4, n = lane & 15;
  const Place at = place_at(blockIdx.x, blockIdx.y, p.xcd != 0, p.linear != 0, p.splits * p.tiles, p.num_kv_heads, p.inv_heads);
  const int s = at.seq, hk = at.head, split = at.split / p.tiles, tile = at.split - split * p.tiles;
  const bool shared = p.max_blocks < 0;  // (the sign says whether a table row is a sequence's or a head's)
  const int max_blocks = shared ? -p.max_blocks : p.max_blocks;
  const int32_t* bt = p.block_table + (int64_t)(shared ? s : at.row) * max_blocks;

  int drafts = p.drafts;
  if (p.draft_lens != nullptr) {
    const int have = p.draft_lens[s];
    drafts = have < 0 ? 0 : have < drafts ? have : drafts;
  }
  const int rows = drafts * p.group, row0 = tile * ROWS;
  if (row0 >= rows) return;
  int len = p.seq_lens[s];
  const int64_t most = (int64_t)max_blocks << p.log2_block;  // (a longer row is a caller error: its table ends here)
  len = len < 0 ? 0 : len < most ? len : (int)most;
  const int cached = len / STEP + (len % STEP != 0), steps = cached + (drafts + STEP - 1) / STEP;
  const int first = split * kWaves + wave, stride = p.splits * kWaves;

  // ---- queries ---------------------------------------------------------------------------------------------------
  const int num_q_heads = p.num_kv_heads * p.group;
  uint4 q[NQ][CH];
  uint64_t sees[NQ];  // drafts that the lane's query row attends to
  const uint64_t real = drafts >= 64 ? ~0ull : (1ull << drafts) - 1;
#pragma unroll
  for (int a = 0; a < NQ; ++a) {
    const int r = row0 + 16 * a + n;
    const int draft = r < rows ? r / p.group : 0, h = r < rows ? r - draft * p.group : 0;
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) +
                                                       (((int64_t)s * p.drafts + draft) * num_q_heads + hk * p.group + h) * D);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      q[a][j] = from[4 * j + g];
      if (r >= rows) q[a][j] = make_uint4(0u, 0u, 0u, 0u);
    }
    sees[a] = r < rows ? p.mask[(int64_t)s * p.drafts + draft] & real : 0ull;
  }

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

  const int64_t token_stride = shared ? (int64_t)p.num_kv_heads * D : D;   // of a page
  const int64_t draft_stride = (int64_t)p.num_kv_heads * D;
  // First token of part `part` of step `step`, as an element offset, and whether it lies in the pools; a part behind the row's
  // end reads its first token again.
  uint4 kb[PARTS][CH];
  uint32_t vb[PARTS][4][VD];
  const auto load = [&](int step, bool keys) {
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const bool pool = step < cached;
      int tok = pool ? step * STEP + part * 16 : (step - cached) * STEP + part * 16;
      const int end = pool ? len : drafts;
      if (tok >= end) tok = 0;
      const void* base;
      int64_t off, stride_t;
      if (pool) {
        int page = bt[tok >> p.log2_block];
        page = page < 0 ? 0 : page;
        off = (((int64_t)page << p.log2_block) + (tok & ((1 << p.log2_block) - 1))) * token_stride + (shared ? hk * D : 0);
        stride_t = token_stride;
        base = keys ? p.k_pool : p.v_pool;
      } else {
        off = ((int64_t)s * p.drafts + tok) * draft_stride + (int64_t)hk * D;
        stride_t = draft_stride;
        base = keys ? p.k_draft : p.v_draft;
      }
      const T* from = static_cast<const T*>(base) + off;
      // (drafts: no token behind the last one is read; a page is read to the end of its 16 tokens)
      const int last = pool ? 15 : drafts - 1 - tok < 15 ? drafts - 1 - tok : 15;
      if (keys) {
        const int t = n < last ? n : last;
#pragma unroll
        for (int j = 0; j < CH; ++j) kb[part][j] = reinterpret_cast<const uint4*>(from + t * stride_t)[4 * j + g];
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = 4 * g + r < last ? 4 * g + r : last;
          const uint32_t* src = reinterpret_cast<const uint32_t*>(from + t * stride_t + n * E);
#pragma unroll
          for (int w = 0; w < VD; w += (VD >= 4 ? 4 : 2)) {
            if constexpr (VD >= 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(src + w);
              vb[part][r][w] = v.x, vb[part][r][w + 1] = v.y, vb[part][r][w + 2] = v.z, vb[part][r][w + 3] = v.w;
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(src + w);
              vb[part][r][w] = v.x, vb[part][r][w + 1] = v.y;
            }
          }
        }
      }
    }
  };

  if (first < steps) {
    load(first, true);
    load(first, false);
  }
  for (int step = first; step < steps; step += stride) {
    const bool pool = step < cached;
    const int tok0 = pool ? step * STEP : (step - cached) * STEP;
    const int end = pool ? len : drafts;
    f32x4_t x[NQ][PARTS];
#pragma unroll
    for (int a = 0; a < NQ; ++a)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        f32x4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
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
        x[a][part] = c * p.scale_log2e;
      }
    const bool more = step + stride < steps;
    if (more) load(step + stride, true);
    if (!pool || tok0 + STEP > len) {
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
            const bool in = pool ? t < len : (t < 64 && ((sees[a] >> (t & 63)) & 1u) != 0);
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
      float sum = 0.f;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[a][part][r] = __builtin_amdgcn_exp2f(x[a][part][r] - m_ref[a]);
          sum += x[a][part][r];
        }
      l_run[a] += sum;
    }
    if constexpr (GE::kBf16) {
      bf16x8_t hi[NQ], lo[NQ];
#pragma unroll
      for (int a = 0; a < NQ; ++a) {
        uint4 h, l;
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t p0 = __float_as_uint(x[a][w / 2][w % 2 * 2]), p1 = __float_as_uint(x[a][w / 2][w % 2 * 2 + 1]);
          hw[w] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
          const float r0 = __uint_as_float(p0) - __uint_as_float(p0 & 0xffff0000u), r1 = __uint_as_float(p1) - __uint_as_float(p1 & 0xffff0000u);
          lw[w] = __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x07060302u);
        }
        h = make_uint4(hw[0], hw[1], hw[2], hw[3]);
        l = make_uint4(lw[0], lw[1], lw[2], lw[3]);
        hi[a] = __builtin_bit_cast(bf16x8_t, h);
        lo[a] = __builtin_bit_cast(bf16x8_t, l);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
        const uint4 t = make_uint4(__builtin_amdgcn_perm(vb[0][1][e >> 1], vb[0][0][e >> 1], sel),
                                   __builtin_amdgcn_perm(vb[0][3][e >> 1], vb[0][2][e >> 1], sel),
                                   __builtin_amdgcn_perm(vb[PARTS - 1][1][e >> 1], vb[PARTS - 1][0][e >> 1], sel),
                                   __builtin_amdgcn_perm(vb[PARTS - 1][3][e >> 1], vb[PARTS - 1][2][e >> 1], sel));
        const bf16x8_t v = __builtin_bit_cast(bf16x8_t, t);
#pragma unroll
        for (int a = 0; a < NQ; ++a) {
          acc[a][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi[a], acc[a][e], 0, 0, 0);
          acc[a][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo[a], acc[a][e], 0, 0, 0);
        }
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
    if (more) load(step + stride, false);
  }

  // ---- the waves' states, 16 query rows at a time ---------------------------------------------------------------------
#pragma unroll
  for (int a = 0; a < NQ; ++a) {
    const float l = rows_sum(l_run[a]);
    if (g == 0) sm_ml[wave][n] = make_float2(m_run[a], l);
    // lane (g, n) has rows 4*g + r of C: elements (4*g + r) * E + e of query n
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(&sm_acc[wave][n][(4 * g + r) * E + e]) =
            make_float4(acc[a][e][r], acc[a][e + 1][r], acc[a][e + 2][r], acc[a][e + 3][r]);
    }
    __syncthreads();
    for (int idx = (int)threadIdx.x; idx < 16 * (D / 2); idx += kWaves * kWave) {
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
      if (p.splits == 1) {
        const int draft = r / p.group, h = r - draft * p.group;
        const int64_t head = ((int64_t)s * p.drafts + draft) * num_q_heads + hk * p.group + h;
        store_pair<T>(p.out, (head * D + d) / 2, lsum > 0.f ? o0 / lsum : 0.f, lsum > 0.f ? o1 / lsum : 0.f);
      } else {
        float* record = p.partials + (((int64_t)at.row * p.splits + split) * (p.drafts * p.group) + r) * (D + 2);
        *reinterpret_cast<float2*>(record + d) = make_float2(o0, o1);
        if (d == 0) *reinterpret_cast<float2*>(record + D) = make_float2(m, lsum);
      }
    }
    if (a + 1 < NQ) __syncthreads();
  }
}

// The splits of a query row, one wave each, added in their order.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * kWave) void tree_merge_kernel(const TreeParams p) {
  constexpr int E = D / kWave;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int most = p.drafts * p.group, tiles = (most + kWaves - 1) / kWaves;
  const int row = (int)(blockIdx.x / (uint32_t)tiles), r = ((int)blockIdx.x - row * tiles) * kWaves + wave;
  const int s = row / p.num_kv_heads, hk = row - s * p.num_kv_heads;
  int drafts = p.drafts;
  if (p.draft_lens != nullptr) {
    const int have = p.draft_lens[s];
    drafts = have < 0 ? 0 : have < drafts ? have : drafts;
  }
  if (r >= drafts * p.group) return;
  const float* base = p.partials + ((int64_t)row * p.splits * most + r) * (D + 2);
  float o[E];
  merge_splits<E>(p.splits, o, [&](int split, float2& ml, float (&v)[E]) {
    const float* record = base + (int64_t)split * most * (D + 2);
    ml = *reinterpret_cast<const float2*>(record + D);
    if constexpr (E == 2) {
      const float2 pair = *reinterpret_cast<const float2*>(record + lane * 2);
      v[0] = pair.x, v[1] = pair.y;
    } else {
      v[0] = record[lane];
    }
  });
  const int draft = r / p.group, h = r - draft * p.group;
  const int64_t to = (((int64_t)s * p.drafts + draft) * (p.num_kv_heads * p.group) + hk * p.group + h) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (sizeof(T) == 4)
      static_cast<float*>(p.out)[to + e] = o[e];
    else
      static_cast<uint16_t*>(p.out)[to + e] = f32_to_bf16(o[e]);
  }
}

template <typename T, int D, int NQ>
hipError_t launch_tiles(const TreeArgs& a, TreeParams p, hipStream_t stream) {
  p.tiles = (a.drafts * p.group + 16 * NQ - 1) / (16 * NQ);
  PlaceGrid grid;
  if (!place_grid(a.num_seqs, a.num_kv_heads, p.splits * p.tiles, true, &grid)) return hipErrorInvalidValue;
  p.xcd = grid.xcd, p.linear = grid.linear, p.inv_heads = grid.inv_heads;
  hipLaunchKernelGGL((tree_decode_kernel<T, D, NQ>), dim3(grid.x, grid.y), dim3(kWaves * kWave), 0, stream, p);
  if (p.splits > 1) {
    const int64_t blocks = (int64_t)a.num_seqs * a.num_kv_heads * ((a.drafts * p.group + kWaves - 1) / kWaves);
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3((unsigned)blocks), dim3(kWaves * kWave), 0, stream, p);
  }
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_rows(const TreeArgs& a, const TreeParams& p, hipStream_t stream) {
  switch (a.tile_rows) {
    case 16: return launch_tiles<T, D, 1>(a, p, stream);
    case 32: return launch_tiles<T, D, 2>(a, p, stream);
    case 64:
      if constexpr (sizeof(T) == 2) return launch_tiles<T, D, 4>(a, p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_tree_decode(const TreeArgs& a, hipStream_t stream) {
  TreeParams p{};
  p.q = a.q, p.k_draft = a.k_draft, p.v_draft = a.v_draft;
  p.draft_lens = a.draft_lens, p.mask = a.mask;
  p.k_pool = a.k_pool, p.v_pool = a.v_pool;
  p.block_table = a.block_table, p.seq_lens = a.seq_lens;
  p.out = a.out, p.partials = a.partials;
  p.scale_log2e = a.scale * 1.4426950408889634f;
  p.num_kv_heads = a.num_kv_heads, p.group = a.num_q_heads / a.num_kv_heads, p.drafts = a.drafts;
  p.max_blocks = a.shared ? -a.max_blocks : a.max_blocks;
  while ((1 << p.log2_block) < a.block_size) ++p.log2_block;
  p.splits = a.splits;
  if (a.is_bf16) return a.head_dim == 64 ? launch_rows<bf16_t, 64>(a, p, stream) : launch_rows<bf16_t, 128>(a, p, stream);
  return a.head_dim == 64 ? launch_rows<float, 64>(a, p, stream) : launch_rows<float, 128>(a, p, stream);
}

}  // namespace pe
