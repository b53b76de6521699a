// Pages whose keys can give the largest products with a query: the bounds of a page's keys, and the choice by them.
//
// Bounds: lo_d and hi_d, the smallest and the largest of a full page's keys in each element d (values of the cache's own type, so
// nothing is rounded).  For any key k of the page q_d k_d <= max(q_d lo_d, q_d hi_d), so the sum of these over the elements, and
// over the query heads that share the row's decision, is no less than any sum of their products with one key.
//
// max(q lo, q hi) = max(q, 0) hi + min(q, 0) lo, whatever the signs (lo <= hi).  So the score of a page, over all its query heads, is
// ONE dot product of 2 D terms: <up, hi> + <down, lo> with up_d = sum_h max(q_hd, 0), down_d = sum_h min(q_hd, 0).  What bounds it is
// reading the bounds (2/B of the cache's keys); the query heads cost nothing per page, and the products can be summed in 64 bits
// (rounded once to fp32), so that the choice does not depend on the order of a sum.
#include "pe_norms.h"
#include "pe_select.h"

namespace pe {
namespace {

constexpr int kWaves = 4;

// ---- bounds --------------------------------------------------------------------------------------------------------------
// One wave a page and head.  A lane's 16 bytes of every TPL-th token, the smallest and largest over its tokens, then over the lanes
// that hold the same elements.
template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  return (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u);
}

template <int FROM, int N>
__device__ __forceinline__ void bounds_over_lanes(float (&lo)[N], float (&hi)[N]) {
  if constexpr (FROM < kWave) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      lo[e] = fminf(lo[e], lane_xor_f32<FROM>(lo[e]));
      hi[e] = fmaxf(hi[e], lane_xor_f32<FROM>(hi[e]));
    }
    bounds_over_lanes<FROM * 2>(lo, hi);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kWaves * kWave) void page_bounds_kernel(const void* k_pool, const int32_t* block_table, const int32_t* seq_lens,
                                                                     void* bounds, int recent, int num_kv_heads, int log2_block, int max_blocks,
                                                                     int shared, int64_t items, int per_row) {
  using Geo = RowGeom<T, D>;
  constexpr int EPL = Geo::kPerVec, LPR = Geo::kLanesPerRow, TPL = Geo::kTokensPerLoad;
  const int lane = lane_id(), u = lane % LPR, grp = lane / LPR;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  for (int64_t item = (int64_t)blockIdx.x * kWaves + wave; item < items; item += (int64_t)gridDim.x * kWaves) {
    const int64_t row = item / per_row;  // (sequence, KV head)
    int j = (int)(item - row * per_row);
    const int s = (int)(row / num_kv_heads), hk = (int)(row - (int64_t)s * num_kv_heads);
    const int len = seq_lens[s];
    int full = len > 0 ? len >> log2_block : 0;
    full = full < max_blocks ? full : max_blocks;
    if (recent > 0) j += full - per_row;
    if (j < 0 || j >= full) continue;
    const int page = block_table[(shared ? s : row) * max_blocks + j];
    if (page < 0) continue;
    const int heads = shared ? num_kv_heads : 1;
    const int64_t first = ((int64_t)page << log2_block) * heads * LPR + (shared ? hk * LPR : 0);
    float lo[EPL], hi[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      lo[e] = __builtin_inff();
      hi[e] = -__builtin_inff();
    }
    for (int t = 0; t < 1 << log2_block; t += 16) {
      uint4 k[16 / TPL];
#pragma unroll
      for (int i = 0; i < 16 / TPL; ++i) k[i] = load_vec_stream(k_pool, first + (int64_t)(t + i * TPL + grp) * heads * LPR + u);
#pragma unroll
      for (int i = 0; i < 16 / TPL; ++i)
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float x = vec_elem<T>(k[i], e);
          lo[e] = fminf(lo[e], x);
          hi[e] = fmaxf(hi[e], x);
        }
    }
    bounds_over_lanes<LPR>(lo, hi);
    if (grp < 2) {
      const float(&v)[EPL] = grp == 0 ? lo : hi;
      uint4 w;
      if constexpr (sizeof(T) == 4)
        w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      else
        w = make_uint4(pack_pair<T>(v[0], v[1]), pack_pair<T>(v[2], v[3]), pack_pair<T>(v[4], v[5]), pack_pair<T>(v[6], v[7]));
      static_cast<uint4*>(bounds)[((int64_t)page * 2 + grp) * heads * LPR + (shared ? hk * LPR : 0) + u] = w;
    }
  }
}

// ---- scores --------------------------------------------------------------------------------------------------------------
// A wave scores 16 * 64 / LPB pages: the 2 D bounds of a page and head are LPB lanes' 16 bytes, lo in the lower half of them and hi in
// the upper.  Sixteen loads are in flight; their sums meet in a reduce-scatter.  Head-shared rows add their heads up before it.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * kWave) void score_pages_kernel(const void* q, const void* bounds, const int32_t* block_table,
                                                                     const int32_t* seq_lens, float* scores, int num_kv_heads, int group,
                                                                     int log2_block, int max_blocks, int shared, int pages, int parts,
                                                                     int64_t first_row) {
  constexpr int EPL = Elem<T>::kPerVec, LPB = 2 * D / EPL, PPL = kWave / LPB, NL = 16, kPages = NL * PPL;
  const int lane = lane_id(), u = lane % LPB, up = u / (LPB / 2), v = u % (LPB / 2);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int64_t row = first_row + blockIdx.x / (uint32_t)parts;  // of the table
  const int part = (int)(blockIdx.x % (uint32_t)parts);
  const int s = (int)(shared ? row : row / num_kv_heads);
  int len = seq_lens[s];
  const int all = len > 0 ? (int)(((int64_t)len + (1 << log2_block) - 1) >> log2_block) : 0;
  const int n = (all < max_blocks ? all : max_blocks) - 1;  // candidates: all but the newest page
  const int base = (part * kWaves + wave) * kPages;
  if (n < pages || base >= n) return;  // (with n + 1 <= pages every page is taken)
  const int32_t* bt = block_table + row * max_blocks;
  const int heads = shared ? num_kv_heads : 1, head0 = shared ? 0 : (int)(row - (int64_t)s * num_kv_heads);
  int64_t at[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int j = base + i * PPL + lane / LPB;
    const int page = bt[j < n ? j : n - 1];
    at[i] = ((int64_t)(page < 0 ? 0 : page) * 2 + up) * heads * (LPB / 2) + v;
  }
  double sum[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) sum[i] = 0.0;
  for (int h = 0; h < heads; ++h) {
    uint4 b[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) b[i] = load_vec(bounds, at[i] + h * (LPB / 2));
    double w[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) w[e] = 0.0;
    const uint4* from = static_cast<const uint4*>(q) + ((int64_t)s * num_kv_heads + head0 + h) * group * (LPB / 2) + v;
    for (int x = 0; x < group; ++x) {
      const uint4 qv = from[x * (LPB / 2)];
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float f = vec_elem<T>(qv, e);
        w[e] += (double)(up ? fmaxf(f, 0.f) : fminf(f, 0.f));
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
      for (int e = 0; e < EPL; ++e) sum[i] = fma((double)vec_elem<T>(b[i], e), w[e], sum[i]);
  }
  double total = reduce_scatter_f64<NL>(sum, lane);  // of load bit_reverse(lane & 15)
  total = all_reduce_f64<NL, LPB>(total);
  const int j = base + bit_reverse<4>(lane & 15) * PPL + lane / LPB;
  if (u < NL && j < n) scores[row * max_blocks + j] = (float)total;
}

// ---- selection -----------------------------------------------------------------------------------------------------------
// One workgroup a row.  Scores as whole numbers in the same order; the smallest one that is taken is found two bits at a time, by
// counting those that reach each of three thresholds; what reaches it is taken, of equal ones the first.
constexpr int kThreads = 1024, kSelectWaves = kThreads / kWave, kHeld = 8;

__device__ __forceinline__ uint32_t order_of(float f) {
  const uint32_t b = __float_as_uint(f + 0.f);  // (-0 is 0)
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kThreads) void select_pages_kernel(const float* scores, const int32_t* block_table, const int32_t* seq_lens,
                                                                int32_t* table_out, int32_t* lens_out, int32_t* idx_out, int num_kv_heads,
                                                                int log2_block, int max_blocks, int shared, int pages, int64_t first_row) {
  __shared__ uint32_t counts[16][4];
  __shared__ uint32_t above[2][kSelectWaves], equal[2][kSelectWaves];
  const int64_t row = first_row + blockIdx.x;
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int s = (int)(shared ? row : row / num_kv_heads);
  const int64_t most = (int64_t)max_blocks << log2_block;
  int len = seq_lens[s];
  len = len < 0 ? 0 : len < most ? len : (int)most;
  const int all = (int)(((int64_t)len + (1 << log2_block) - 1) >> log2_block);
  const int taken = all < pages ? all : pages;
  const int32_t* bt = block_table + row * max_blocks;
  int32_t* to = table_out + row * pages;
  int32_t* idx = idx_out != nullptr ? idx_out + row * pages : nullptr;
  for (int i = taken + tid; i < pages; i += kThreads) {
    to[i] = -1;
    if (idx != nullptr) idx[i] = -1;
  }
  if (tid == 0 && (shared || row == (int64_t)s * num_kv_heads)) lens_out[s] = len - ((all - taken) << log2_block);
  if (all <= pages) {
    for (int i = tid; i < all; i += kThreads) {
      to[i] = bt[i];
      if (idx != nullptr) idx[i] = i;
    }
    return;
  }
  const int n = all - 1, need = pages - 1;  // need < n
  if (tid == 0) {
    to[need] = bt[n];
    if (idx != nullptr) idx[need] = n;
  }
  if (need == 0) return;
  const float* sc = scores + row * max_blocks;
  const int rounds = (n + kThreads - 1) / kThreads;
  uint32_t held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = i * kThreads + tid < n ? order_of(sc[i * kThreads + tid]) : 0u;
  if (tid < 64) counts[tid / 4][tid % 4] = 0u;
  __syncthreads();
  uint32_t least = 0u;
  for (int bit = 30, at = 0; bit >= 0; bit -= 2, ++at) {
    uint32_t c[3] = {0u, 0u, 0u};
    const auto count = [&](uint32_t key) {
#pragma unroll
      for (int t = 0; t < 3; ++t) c[t] += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= least + ((uint32_t)(t + 1) << bit)));
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < rounds) count(held[i]);
    for (int i = kHeld; i < rounds; ++i) {
      const int j = i * kThreads + tid;
      count(j < n ? order_of(sc[j]) : 0u);
    }
    if (lane < 3) atomicAdd(&counts[at][lane], lane == 0 ? c[0] : lane == 1 ? c[1] : c[2]);
    __syncthreads();
    uint32_t step = 0u;
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (counts[at][t] >= (uint32_t)need) step = (uint32_t)(t + 1) << bit;
    least += step;
  }
  // what lies above is counted again, to know how many of the equal ones go
  __shared__ uint32_t over;
  if (tid == 0) over = 0u;
  __syncthreads();
  uint32_t c = 0u;
  for (int i = 0; i < rounds; ++i) {
    const int j = i * kThreads + tid;
    c += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(j < n && order_of(sc[j]) > least));
  }
  if (lane == 0) atomicAdd(&over, c);
  __syncthreads();
  const int ties = need - (int)over;  // the first of the equal ones
  int at_above = 0, at_equal = 0;
  const uint64_t below = (1ull << lane) - 1;
  for (int i = 0; i < rounds; ++i) {
    const int j = i * kThreads + tid;
    const uint32_t key = j < n ? order_of(sc[j]) : 0u;
    const uint64_t gt = __builtin_amdgcn_ballot_w64(j < n && key > least), eq = __builtin_amdgcn_ballot_w64(j < n && key == least);
    if (lane == 0) {
      above[i & 1][wave] = (uint32_t)__builtin_popcountll(gt);
      equal[i & 1][wave] = (uint32_t)__builtin_popcountll(eq);
    }
    __syncthreads();
    int my_above = at_above, my_equal = at_equal;
    for (int w = 0; w < kSelectWaves; ++w) {
      const int a = (int)above[i & 1][w], e = (int)equal[i & 1][w];
      if (w < wave) {
        my_above += a;
        my_equal += e;
      }
      at_above += a;
      at_equal += e;
    }
    my_above += (int)__builtin_popcountll(gt & below);
    my_equal += (int)__builtin_popcountll(eq & below);
    const bool is_gt = (gt >> lane & 1u) != 0, is_eq = (eq >> lane & 1u) != 0 && my_equal < ties;
    if (is_gt || is_eq) {
      const int pos = my_above + (my_equal < ties ? my_equal : ties);
      to[pos] = bt[j];
      if (idx != nullptr) idx[pos] = j;
    }
  }
}

template <typename T, int D>
hipError_t launch_bounds_as(const BoundsArgs& a, hipStream_t stream) {
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const int per_row = a.recent > 0 && a.recent < a.max_blocks ? a.recent : a.max_blocks;
  const int64_t items = (int64_t)a.num_seqs * a.num_kv_heads * per_row;
  const int64_t groups = (items + kWaves - 1) / kWaves;
  hipLaunchKernelGGL((page_bounds_kernel<T, D>), dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(kWaves * kWave), 0, stream, a.k_pool,
                     a.block_table, a.seq_lens, a.bounds, a.recent > 0 ? per_row : 0, a.num_kv_heads, log2_block, a.max_blocks, a.shared ? 1 : 0,
                     items, per_row);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_select_as(const SelectArgs& a, hipStream_t stream) {
  constexpr int kPages = kWaves * 16 * kWave / (2 * D / Elem<T>::kPerVec);  // of a workgroup
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const int64_t rows = a.shared ? a.num_seqs : (int64_t)a.num_seqs * a.num_kv_heads;
  const int group = a.num_q_heads / a.num_kv_heads, parts = (a.max_blocks + kPages - 1) / kPages;
  if (a.max_blocks > a.pages && a.pages > 1) {
    const int64_t some = ((1LL << 32) - 1) / (kWaves * kWave) / parts;  // rows of a launch (of fewer than 2^32 threads)
    if (some < 1) return hipErrorInvalidValue;
    for (int64_t row = 0; row < rows; row += some) {
      const int64_t now = rows - row < some ? rows - row : some;
      hipLaunchKernelGGL((score_pages_kernel<T, D>), dim3((unsigned)(now * parts)), dim3(kWaves * kWave), 0, stream, a.q, a.bounds, a.block_table,
                         a.seq_lens, a.scores, a.num_kv_heads, group, log2_block, a.max_blocks, a.shared ? 1 : 0, a.pages, parts, row);
    }
  }
  constexpr int64_t kRows = 1 << 21;
  for (int64_t row = 0; row < rows; row += kRows)
    hipLaunchKernelGGL(select_pages_kernel, dim3((unsigned)(rows - row < kRows ? rows - row : kRows)), dim3(kThreads), 0, stream, a.scores,
                       a.block_table, a.seq_lens, a.table_out, a.lens_out, a.idx_out, a.num_kv_heads, log2_block, a.max_blocks,
                       a.shared ? 1 : 0, a.pages, row);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_bounds(const BoundsArgs& a, hipStream_t stream) {
  if (a.is_bf16) return a.head_dim == 64 ? launch_bounds_as<bf16_t, 64>(a, stream) : launch_bounds_as<bf16_t, 128>(a, stream);
  return a.head_dim == 64 ? launch_bounds_as<float, 64>(a, stream) : launch_bounds_as<float, 128>(a, stream);
}

hipError_t launch_select_pages(const SelectArgs& a, hipStream_t stream) {
  if (a.is_bf16) return a.head_dim == 64 ? launch_select_as<bf16_t, 64>(a, stream) : launch_select_as<bf16_t, 128>(a, stream);
  return a.head_dim == 64 ? launch_select_as<float, 64>(a, stream) : launch_select_as<float, 128>(a, stream);
}

}  // namespace pe
