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
static_assert(kWaves * kWave == kBoundsThreads && kWaves * kWave == kScoreThreads, "what the host counts with");

// ---- bounds --------------------------------------------------------------------------------------------------------------
// A lane has 16 bytes of every token of one page (head-shared: of one head too), so nothing is exchanged between lanes, and the lanes of
// a wave read whole token rows.  Sixteen loads are in flight.  Bound by the memory: 16 sequences of 8000 to 16384 tokens, eight heads of
// D = 128, pages of 32, head-shared, bfloat16 (400 MB of keys, 25 MB of bounds) 76 us.  Without its stores it takes 61 (6.6 TB/s), and they
// take as long past the caches or through them; more loads in flight, several pages a lane or another order of the workgroups change nothing.
// A page of each of 64 rows takes 3 to 4 us, the launch.
__device__ __forceinline__ uint32_t pack_pair(float a, float b) { return (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u); }

template <typename T>
__global__ __launch_bounds__(kWaves * kWave) void page_bounds_kernel(const uint4* k_pool, const int32_t* block_table, const int32_t* seq_lens,
                                                                     uint4* bounds, int chunks, int rows_per_seq, int log2_block, int max_blocks,
                                                                     int per_row, int groups, int recent, int64_t first_row) {
  constexpr int EPL = Elem<T>::kPerVec;
  const uint32_t in = blockIdx.x / (uint32_t)groups;
  const int64_t row = first_row + in;  // of the table
  const uint32_t unit = (blockIdx.x - in * (uint32_t)groups) * (kWaves * kWave) + threadIdx.x;  // (page, chunk of its token rows)
  int j = (int)(unit / (uint32_t)chunks);
  const int c = (int)(unit - (uint32_t)j * (uint32_t)chunks);
  const int len = seq_lens[(uint32_t)row / (uint32_t)rows_per_seq];
  if (j >= per_row) return;
  int page;
  if (recent) {
    const int full = len > 0 ? len >> log2_block : 0;
    j += (full < max_blocks ? full : max_blocks) - per_row;
    if (j < 0) return;
    page = block_table[row * max_blocks + j];
  } else {  // (the length and the page travel together)
    page = block_table[row * max_blocks + j];
    if (len >> log2_block <= j) return;
  }
  if (page < 0) return;
  const uint4* from = k_pool + (((int64_t)page << log2_block) * chunks + c);
  float lo[EPL], hi[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    lo[e] = __builtin_inff();
    hi[e] = -__builtin_inff();
  }
  for (int t = 0; t < 1 << log2_block; t += 16) {
    uint4 k[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) k[i] = load_vec_stream(from, (int64_t)(t + i) * chunks);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float x = vec_elem<T>(k[i], e);
        lo[e] = fminf(lo[e], x);
        hi[e] = fmaxf(hi[e], x);
      }
  }
  uint4* to = bounds + ((int64_t)page * 2 * chunks + c);
  if constexpr (sizeof(T) == 4) {
    to[0] = make_uint4(__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(lo[2]), __float_as_uint(lo[3]));
    to[chunks] = make_uint4(__float_as_uint(hi[0]), __float_as_uint(hi[1]), __float_as_uint(hi[2]), __float_as_uint(hi[3]));
  } else {
    to[0] = make_uint4(pack_pair(lo[0], lo[1]), pack_pair(lo[2], lo[3]), pack_pair(lo[4], lo[5]), pack_pair(lo[6], lo[7]));
    to[chunks] = make_uint4(pack_pair(hi[0], hi[1]), pack_pair(hi[2], hi[3]), pack_pair(hi[4], hi[5]), pack_pair(hi[6], hi[7]));
  }
}

// ---- scores --------------------------------------------------------------------------------------------------------------
// A wave scores NL * 64 / LPB pages at a time: the 2 D bounds of a page and head are LPB lanes' 16 bytes, lo in the lower half of them and hi
// in the upper.  NL loads are in flight; their sums meet in a reduce-scatter.  4 sequences of 60001 to 65536 tokens (32 rows of 4096 pages,
// 64 MB of bounds) take 14 us: ten at the rate of a large read, then the launch, and the way from the length to the pages to their bounds.
template <typename T, int D, int NL>
struct Scorer {
  static constexpr int EPL = Elem<T>::kPerVec, LPB = 2 * D / EPL, PPL = kWave / LPB, kPages = NL * PPL;

  // The page (behind `base`) whose score the lane is left with, if it is left with one.
  static __device__ __forceinline__ int page_of(int lane) { return bit_reverse<ilog2(NL)>(lane & (NL - 1)) * PPL + lane / LPB; }
  static __device__ __forceinline__ bool has_page(int lane) { return lane % LPB < NL; }
  // The pages of a lane's parts, as the table has them up to entry `last`.
  static __device__ __forceinline__ void look_up(const int32_t* bt, int base, int last, int lane, int32_t (&page)[NL]) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int j = base + i * PPL + lane / LPB;
      page[i] = bt[j < last ? j : last];
    }
  }

  // Scores of those of them that are candidates (below n), over the heads head, head + step, ... of the row's `heads` (first of them:
  // q_head).  In the others' place page 0 is read: their scores go nowhere.
  static __device__ __forceinline__ double score(const uint4* q, const uint4* bounds, const int32_t (&page)[NL], int base, int n, int64_t q_head,
                                                 int group, int heads, int head, int step, int lane) {
    const int u = lane % LPB, up = u / (LPB / 2), v = u % (LPB / 2);
    double sum[NL];
    int64_t at[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      sum[i] = 0.0;
      at[i] = ((int64_t)(base + i * PPL + lane / LPB < n && page[i] > 0 ? page[i] : 0) * 2 + up) * heads * (LPB / 2) + v;
    }
    for (int h = head; h < heads; h += step) {
      uint4 b[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) b[i] = load_vec(bounds, at[i] + h * (LPB / 2));
      double w[EPL];
#pragma unroll
      for (int e = 0; e < EPL; ++e) w[e] = 0.0;
      const uint4* from = q + (q_head + h) * group * (LPB / 2) + v;
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
    return all_reduce_f64<NL, LPB>(reduce_scatter_f64<NL>(sum, lane));
  }
};

struct Row {  // of the table
  int64_t row;
  int s, len, all;  // its sequence, tokens, pages
};
__device__ __forceinline__ Row row_at(int64_t row, const int32_t* seq_lens, int rows_per_seq, int log2_block, int max_blocks) {
  Row r;
  r.row = row;
  r.s = (int)((uint32_t)row / (uint32_t)rows_per_seq);
  const int64_t most = (int64_t)max_blocks << log2_block;
  const int len = seq_lens[r.s];
  r.len = len < 0 ? 0 : len < most ? len : (int)most;
  r.all = (int)(((int64_t)r.len + (1 << log2_block) - 1) >> log2_block);
  return r;
}

// Scores of a row's pages but the newest, for a launch behind this one.  A workgroup has its four waves' pages, or with several heads a
// decision (HEADS) those of one wave, of which each wave takes every fourth head.
template <typename T, int D, int NL, bool HEADS>
__global__ __launch_bounds__(kWaves * kWave, NL == 16 ? 4 : 1) void score_pages_kernel(
    const uint4* q, const uint4* bounds, const int32_t* block_table, const int32_t* seq_lens, float* scores, int rows_per_seq, int heads, int group,
    int log2_block, int max_blocks, int pages, int parts, int64_t first_row) {
  using SC = Scorer<T, D, NL>;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const uint32_t in = blockIdx.x / (uint32_t)parts;
  const int part = (int)(blockIdx.x - in * (uint32_t)parts);
  const int base = (HEADS ? part : part * kWaves + wave) * SC::kPages;
  if (base >= max_blocks) return;
  int32_t page[NL];
  SC::look_up(block_table + (first_row + in) * max_blocks, base, max_blocks - 1, lane, page);  // (they travel together with the length)
  const Row r = row_at(first_row + in, seq_lens, rows_per_seq, log2_block, max_blocks);
  const int n = r.all - 1;  // candidates
  if (n < pages || base >= n) return;  // (with n + 1 <= pages every page is taken; several heads: the same in all waves)
  const int j = base + SC::page_of(lane);
  float* to = scores + r.row * max_blocks + j;
  const bool mine = SC::has_page(lane) && j < n;
  if constexpr (!HEADS) {
    const double total = SC::score(q, bounds, page, base, n, r.row, group, 1, 0, 1, lane);
    if (mine) *to = (float)total;
  } else {
    __shared__ double of_heads[kWaves][kWave];
    of_heads[wave][lane] = SC::score(q, bounds, page, base, n, r.row * heads, group, heads, wave, kWaves, lane);
    __syncthreads();
    if (wave != 0 || !mine) return;
    double total = of_heads[0][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) total += of_heads[w][lane];
    *to = (float)total;
  }
}

// ---- selection -----------------------------------------------------------------------------------------------------------
// One workgroup a row.  Scores as whole numbers in the same order; the smallest one that is taken lies in one of 1024 equal parts of their
// range, and there in one of 1024 parts of that, and so on: a count of each part in LDS, then the part in which the sum from above
// reaches what is needed.  (Scores of about the same size differ in their low bits alone: parts of their range hold about as many each,
// digits of the numbers would not.)  A wave holds consecutive pages, so that one exchange tells where its first one goes.  4096 pages of 32
// rows take 10 us in sixteen waves (and in eight), of which 2 to read the scores, 1.8 and 2.4 for the two counts that are needed as a rule and
// 2 to write; 512 pages 6 us in four waves.
constexpr int kParts = 1024, kHeld = 8, kShort = kHeld * kWave;

__device__ __forceinline__ uint32_t order_of(float f) {
  const uint32_t b = __float_as_uint(f + 0.f);  // (-0 is 0)
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
// Over the lanes of a wave, in every lane.
template <typename F>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, F f) {
  v = f(v, dpp_u32<0xB1>(v));    // quad_perm [1,0,3,2]
  v = f(v, dpp_u32<0x4E>(v));    // quad_perm [2,3,0,1]
  v = f(v, dpp_u32<0x124>(v));   // row_ror:4
  v = f(v, dpp_u32<0x128>(v));   // row_ror:8
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(r[0], r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(h[0], h[1]);
}

template <int WAVES>
struct SelectState {
  alignas(16) uint32_t count[2][kParts];  // part p at place_of(p)
  alignas(16) uint32_t lo[WAVES], hi[WAVES];
  int above[WAVES], equal[WAVES];
};

// Lane l has the parts from 1023 - 16 l down, in four reads that its neighbours' lie beside.
__device__ __forceinline__ uint32_t place_of(uint32_t part) { return (part & 12u) << 6 | (63u - (part >> 4)) << 2 | (part & 3u); }

// Of n scores the `need` < n highest (of equal ones the first), in their order: table entries and indices.
template <int WAVES>
__device__ __forceinline__ void select_row(const float* sc, int n, int need, const int32_t* bt, int32_t* to, int32_t* idx, SelectState<WAVES>& sm) {
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int each = (n + WAVES * kWave - 1) / (WAVES * kWave), first = wave * each * kWave + lane;  // of `each` times 64
  uint32_t held[kHeld];
  int32_t page[kHeld];
  uint32_t lo = ~0u, hi = 0u;
  const auto at = [&](int i) { return first + i * kWave; };
  const auto key = [&](int i) { return at(i) < n ? order_of(sc[at(i)]) : 0u; };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const bool in = i < each && at(i) < n;
    page[i] = in ? bt[at(i)] : -1;
    held[i] = in ? order_of(sc[at(i)]) : 0u;
    lo = in && held[i] < lo ? held[i] : lo;
    hi = in && held[i] > hi ? held[i] : hi;
  }
  for (int i = kHeld; i < each; ++i)
    if (at(i) < n) {
      const uint32_t k = key(i);
      lo = k < lo ? k : lo;
      hi = k > hi ? k : hi;
    }
  lo = over_wave(lo, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
  hi = over_wave(hi, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  if (lane == 0) {
    sm.lo[wave] = lo;
    sm.hi[wave] = hi;
  }
  for (int i = tid; i < 2 * kParts; i += WAVES * kWave) sm.count[0][i] = 0u;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    lo = sm.lo[w] < lo ? sm.lo[w] : lo;
    hi = sm.hi[w] > hi ? sm.hi[w] : hi;
  }
  // Keys above `least` go, and `ties` of those that are equal to it.
  uint32_t least = lo;
  int ties = need;
  for (int turn = 0; hi != lo; ++turn) {
    uint32_t* count = sm.count[turn & 1];
    const uint32_t range = hi - lo;
    const int bits = 32 - __builtin_clz(range), shift = bits > 10 ? bits - 10 : 0;
    const auto add = [&](uint32_t k) {
      if (k - lo <= range) atomicAdd(&count[place_of((k - lo) >> shift)], 1u);
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < each && at(i) < n) add(held[i]);
    for (int i = kHeld; i < each; ++i)
      if (at(i) < n) add(key(i));
    __syncthreads();
    // every wave finds the same part
    uint32_t part[16], sum = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 c = *reinterpret_cast<const uint4*>(&count[i * 256 + lane * 4]);
      part[4 * i] = c.x, part[4 * i + 1] = c.y, part[4 * i + 2] = c.z, part[4 * i + 3] = c.w;
      sum += (c.x + c.y) + (c.z + c.w);
    }
    const uint32_t upto = wave_prefix_sum_u32(sum);
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto >= (uint32_t)ties));  // (all of the range are `ties` at least)
    uint32_t over = upto - sum, found = 0u, inside = 0u;
    bool open = true;
#pragma unroll
    for (int i = 15; i >= 0; --i) {
      const bool here = open && over + part[i] >= (uint32_t)ties;
      if (here) {
        found = (uint32_t)(kParts - 16 * (lane + 1) + i);
        inside = part[i];
        open = false;
      }
      if (open) over += part[i];
    }
    found = (uint32_t)__builtin_amdgcn_readlane((int)found, owner);
    inside = (uint32_t)__builtin_amdgcn_readlane((int)inside, owner);
    ties -= __builtin_amdgcn_readlane((int)over, owner);
    lo += found << shift;
    least = lo;
    if (inside == (uint32_t)ties) {  // all of it go: it is no lowest part (need < n), so there is a number below
      least = lo - 1u;
      ties = 0;
      break;
    }
    if (shift == 0) break;
    hi = lo + ((1u << shift) - 1u);
    for (int i = tid; i < kParts; i += WAVES * kWave) sm.count[(turn & 1) ^ 1][i] = 0u;
    __syncthreads();
  }
  int above = 0, equal = 0;
  const auto both = [&](int i, uint32_t k) {
    above += (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(at(i) < n && k > least));
    equal += (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(at(i) < n && k == least));
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (i < each) both(i, held[i]);
  for (int i = kHeld; i < each; ++i) both(i, key(i));
  if (lane == 0) {
    sm.above[wave] = above;
    sm.equal[wave] = equal;
  }
  __syncthreads();
  above = equal = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (w < wave) {
      above += sm.above[w];
      equal += sm.equal[w];
    }
  const uint64_t below = (1ull << lane) - 1;
  const auto put = [&](int i, uint32_t k, int32_t entry) {
    const uint64_t gt = __builtin_amdgcn_ballot_w64(at(i) < n && k > least), eq = __builtin_amdgcn_ballot_w64(at(i) < n && k == least);
    const int before = equal + (int)__builtin_popcountll(eq & below);
    if ((gt >> lane & 1u) != 0 || ((eq >> lane & 1u) != 0 && before < ties)) {
      const int pos = above + (int)__builtin_popcountll(gt & below) + (before < ties ? before : ties);
      to[pos] = entry;
      if (idx != nullptr) idx[pos] = at(i);
    }
    above += (int)__builtin_popcountll(gt);
    equal += (int)__builtin_popcountll(eq);
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (i < each) put(i, held[i], page[i]);
  for (int i = kHeld; i < each; ++i) put(i, key(i), at(i) < n ? bt[at(i)] : -1);
}

__device__ __forceinline__ void entries_of(const int32_t* bt, int n, int32_t (&entry)[kHeld]) {
  const int lane = lane_id();
#pragma unroll
  for (int i = 0; i < kHeld; ++i) entry[i] = i * kWave + lane < n ? bt[i * kWave + lane] : -1;
}

// The same of at most kShort scores, by one wave and without a barrier: the smallest one that is taken by halving the range, a
// ballot for every 64 scores and turn (about log2 n turns and a few more, as it ends where a half's count is right).  2 us for 255 scores
// in LDS where eight waves that count take 3; behind a launch that made the scores, score launch included, one wave / four: 64 pages
// 9.6 / 10.5 us, 256 10.9 / 11.8, 512 12.9 / 12.1.
__device__ __forceinline__ void select_short_row(const float* sc, int n, int need, const int32_t (&page)[kHeld], int32_t* to, int32_t* idx) {
  const int lane = lane_id(), each = (n + kWave - 1) / kWave;
  uint32_t held[kHeld], lo = ~0u, hi = 0u;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const bool in = i * kWave + lane < n;
    held[i] = in ? order_of(sc[i * kWave + lane]) : 0u;
    lo = in && held[i] < lo ? held[i] : lo;
    hi = in && held[i] > hi ? held[i] : hi;
  }
  lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)over_wave(lo, [](uint32_t a, uint32_t b) { return a < b ? a : b; }));
  hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)over_wave(hi, [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
  const auto above = [&](uint32_t least) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) c += (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(held[i] > least));
    return c;
  };
  int ties = need;
  while (lo != hi) {  // fewer than `need` are above hi, and `need` or more are lo or above
    const uint32_t mid = lo + (hi - lo) / 2;
    const int c = above(mid);
    if (c == need) {
      lo = mid;
      break;
    }
    if (c > need)
      lo = mid + 1;
    else
      hi = mid;
  }
  ties -= above(lo);
  int pos = 0, equal = 0;  // taken, and equal ones met, in what lies before
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    if (i >= each) break;
    const bool in = i * kWave + lane < n;
    const uint64_t gt = __builtin_amdgcn_ballot_w64(in && held[i] > lo), eq = __builtin_amdgcn_ballot_w64(in && held[i] == lo);
    const uint64_t below = (1ull << lane) - 1;
    const int before = equal + (int)__builtin_popcountll(eq & below);
    const uint64_t take = gt | __builtin_amdgcn_ballot_w64((eq >> lane & 1u) != 0 && before < ties);
    if (take >> lane & 1u) {
      const int at = pos + (int)__builtin_popcountll(take & below);
      to[at] = page[i];
      if (idx != nullptr) idx[at] = i * kWave + lane;
    }
    pos += (int)__builtin_popcountll(take);
    equal += (int)__builtin_popcountll(eq);
  }
}

// What of a row's outputs does not depend on scores; true if that is everything.
template <int WAVES>
__device__ __forceinline__ bool frame_row(const Row& r, const int32_t* bt, int32_t* to, int32_t* idx, int32_t* lens_out, bool first_head,
                                          int log2_block, int pages) {
  const int tid = (int)threadIdx.x, taken = r.all < pages ? r.all : pages;
  for (int i = taken + tid; i < pages; i += WAVES * kWave) {
    to[i] = -1;
    if (idx != nullptr) idx[i] = -1;
  }
  if (tid == 0 && first_head) lens_out[r.s] = r.len - ((r.all - taken) << log2_block);
  if (r.all <= pages) {
    for (int i = tid; i < r.all; i += WAVES * kWave) {
      to[i] = bt[i];
      if (idx != nullptr) idx[i] = i;
    }
    return true;
  }
  if (tid == 0) {  // the newest
    to[pages - 1] = bt[r.all - 1];
    if (idx != nullptr) idx[pages - 1] = r.all - 1;
  }
  return pages == 1;
}

template <int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void select_pages_kernel(const float* scores, const int32_t* block_table, const int32_t* seq_lens,
                                                                     int32_t* table_out, int32_t* lens_out, int32_t* idx_out, int rows_per_seq,
                                                                     int log2_block, int max_blocks, int pages, int64_t first_row) {
  const Row r = row_at(first_row + blockIdx.x, seq_lens, rows_per_seq, log2_block, max_blocks);
  const int32_t* bt = block_table + r.row * max_blocks;
  int32_t *to = table_out + r.row * pages, *idx = idx_out != nullptr ? idx_out + r.row * pages : nullptr;
  if (frame_row<WAVES>(r, bt, to, idx, lens_out, r.row == (int64_t)r.s * rows_per_seq, log2_block, pages)) return;
  if constexpr (WAVES == 1) {
    int32_t entry[kHeld];
    entries_of(bt, r.all - 1, entry);
    select_short_row(scores + r.row * max_blocks, r.all - 1, pages - 1, entry, to, idx);
  } else {
    __shared__ SelectState<WAVES> sm;
    select_row<WAVES>(scores + r.row * max_blocks, r.all - 1, pages - 1, bt, to, idx, sm);
  }
}

// Scores and selection in one launch, for rows of one head that one workgroup reads soon enough.  (bf16, 32 query heads over 8, one launch /
// two: 1 sequence with 16 KiB of bounds a row 5.6 / 8.4 us, with 64 KiB 7.1 / 9.3, with 128 KiB 9.7 / 9.9, with 256 KiB 16.1 / 10.4; 32
// sequences 6.4 / 9.4, 9.3 / 12.4, 13.5 / 16.4 and 22.6 / 24.8.  Eight heads a decision, 64 pages of 128 KiB: 14.1 / 10.5, as a wave would
// have to take one head after the other.)
constexpr int64_t kOneLaunchBytes = 128 << 10;

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void score_select_kernel(const uint4* q, const uint4* bounds, const int32_t* block_table,
                                                                     const int32_t* seq_lens, int32_t* table_out, int32_t* lens_out,
                                                                     int32_t* idx_out, int rows_per_seq, int group, int log2_block,
                                                                     int max_blocks, int pages, int64_t first_row) {
  using SC = Scorer<T, D, 8>;
  __shared__ float sc[kShort];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const Row r = row_at(first_row + blockIdx.x, seq_lens, rows_per_seq, log2_block, max_blocks);
  const int32_t* bt = block_table + r.row * max_blocks;
  int32_t *to = table_out + r.row * pages, *idx = idx_out != nullptr ? idx_out + r.row * pages : nullptr;
  if (frame_row<WAVES>(r, bt, to, idx, lens_out, r.row == (int64_t)r.s * rows_per_seq, log2_block, pages)) return;
  const int n = r.all - 1;
  int32_t entry[kHeld];
  if (wave == 0) entries_of(bt, n, entry);
  for (int base = wave * SC::kPages; base < n; base += WAVES * SC::kPages) {
    int32_t page[8];
    SC::look_up(bt, base, n - 1, lane, page);
    const double total = SC::score(q, bounds, page, base, n, r.row, group, 1, 0, 1, lane);
    const int j = base + SC::page_of(lane);
    if (SC::has_page(lane) && j < n) sc[j] = (float)total;
  }
  __syncthreads();
  if (wave == 0) select_short_row(sc, n, pages - 1, entry, to, idx);
}

template <typename T>
hipError_t launch_bounds_as(const BoundsArgs& a, hipStream_t stream) {
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const int rows_per_seq = a.shared ? 1 : a.num_kv_heads;
  const int chunks = a.head_dim * (int)sizeof(T) / 16 * (a.shared ? a.num_kv_heads : 1);
  const int per_row = bounds_per_row(a.recent, a.max_blocks);
  const int64_t rows = (int64_t)a.num_seqs * rows_per_seq, groups = bounds_groups(per_row, chunks);
  const int64_t some = ((1LL << 32) - 1) / (kWaves * kWave) / groups;  // rows of a launch (of fewer than 2^32 threads)
  if (some < 1) return hipErrorInvalidValue;
  for (int64_t row = 0; row < rows; row += some) {
    const int64_t now = rows - row < some ? rows - row : some;
    hipLaunchKernelGGL((page_bounds_kernel<T>), dim3((unsigned)(now * groups)), dim3(kWaves * kWave), 0, stream, (const uint4*)a.k_pool,
                       a.block_table, a.seq_lens, (uint4*)a.bounds, chunks, rows_per_seq, log2_block, a.max_blocks, per_row, (int)groups,
                       a.recent > 0 ? 1 : 0, row);
  }
  return hipGetLastError();
}

template <int WAVES>
void launch_select_of(const SelectArgs& a, int rows_per_seq, int log2_block, int64_t rows, hipStream_t stream) {
  constexpr int64_t kRows = 1 << 21;  // of a launch (of fewer than 2^32 threads)
  for (int64_t row = 0; row < rows; row += kRows)
    hipLaunchKernelGGL((select_pages_kernel<WAVES>), dim3((unsigned)(rows - row < kRows ? rows - row : kRows)), dim3(WAVES * kWave), 0, stream,
                       a.scores, a.block_table, a.seq_lens, a.table_out, a.lens_out, a.idx_out, rows_per_seq, log2_block, a.max_blocks, a.pages,
                       row);
}

template <typename T, int D, int NL, bool HEADS>
hipError_t launch_scores(const SelectArgs& a, int rows_per_seq, int heads, int group, int log2_block, int64_t rows, hipStream_t stream) {
  constexpr int64_t kEach = Scorer<T, D, NL>::kPages * (HEADS ? 1 : kWaves);
  static_assert(kEach >= kFewestScored, "what the host counts with");
  const int64_t parts = (a.max_blocks + kEach - 1) / kEach;
  const int64_t some = ((1LL << 32) - 1) / (kWaves * kWave) / parts;
  if (some < 1) return hipErrorInvalidValue;
  for (int64_t row = 0; row < rows; row += some) {
    const int64_t now = rows - row < some ? rows - row : some;
    hipLaunchKernelGGL((score_pages_kernel<T, D, NL, HEADS>), dim3((unsigned)(now * parts)), dim3(kWaves * kWave), 0, stream, (const uint4*)a.q,
                       (const uint4*)a.bounds, a.block_table, a.seq_lens, a.scores, rows_per_seq, heads, group, log2_block, a.max_blocks,
                       a.pages, (int)parts, row);
  }
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_select_as(const SelectArgs& a, hipStream_t stream) {
  int log2_block = 0;
  while ((1 << log2_block) < a.block_size) ++log2_block;
  const int rows_per_seq = a.shared ? 1 : a.num_kv_heads, heads = a.shared ? a.num_kv_heads : 1;
  const int64_t rows = (int64_t)a.num_seqs * rows_per_seq;
  const int group = a.num_q_heads / a.num_kv_heads;
  constexpr int64_t kRows = 1 << 21;
  if (heads == 1 && a.max_blocks <= kShort && (int64_t)a.max_blocks * 2 * D * (int64_t)sizeof(T) <= kOneLaunchBytes) {
    for (int64_t row = 0; row < rows; row += kRows)
      hipLaunchKernelGGL((score_select_kernel<T, D, 8>), dim3((unsigned)(rows - row < kRows ? rows - row : kRows)), dim3(8 * kWave),
                         0, stream, (const uint4*)a.q, (const uint4*)a.bounds, a.block_table, a.seq_lens,
                         a.table_out, a.lens_out, a.idx_out, rows_per_seq, group, log2_block, a.max_blocks, a.pages, row);
    return hipGetLastError();
  }
  if (a.max_blocks > a.pages && a.pages > 1) {
    static_assert(Scorer<T, D, 16>::kPages * kWaves == scored_by_sixteen(D, sizeof(T) == 2), "what the rule counts with");
    hipError_t e;
    if (heads > 1)
      e = launch_scores<T, D, 8, true>(a, rows_per_seq, heads, group, log2_block, rows, stream);
    else if (many_scores(rows, a.max_blocks, D, a.is_bf16, host::compute_units()))
      e = launch_scores<T, D, 16, false>(a, rows_per_seq, heads, group, log2_block, rows, stream);
    else
      e = launch_scores<T, D, 8, false>(a, rows_per_seq, heads, group, log2_block, rows, stream);
    if (e != hipSuccess) return e;
  }
  if (a.max_blocks <= kShort / 2)
    launch_select_of<1>(a, rows_per_seq, log2_block, rows, stream);
  else if (a.max_blocks <= 4 * kWave * kHeld)
    launch_select_of<4>(a, rows_per_seq, log2_block, rows, stream);
  else
    launch_select_of<16>(a, rows_per_seq, log2_block, rows, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_bounds(const BoundsArgs& a, hipStream_t stream) {
  return a.is_bf16 ? launch_bounds_as<bf16_t>(a, stream) : launch_bounds_as<float>(a, stream);
}

hipError_t launch_select_pages(const SelectArgs& a, hipStream_t stream) {
  if (a.is_bf16) return a.head_dim == 64 ? launch_select_as<bf16_t, 64>(a, stream) : launch_select_as<bf16_t, 128>(a, stream);
  return a.head_dim == 64 ? launch_select_as<float, 64>(a, stream) : launch_select_as<float, 128>(a, stream);
}

}  // namespace pe
