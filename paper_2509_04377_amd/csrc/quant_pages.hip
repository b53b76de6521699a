// Pages of a cache rounded to e4m3 (pe_quant_pages), and a decode step's new token, with the page that it fills (pe_quant_append).
//
// A page of a head is read once into registers, by as many waves as hold it (kLoads 16-byte loads of K and of V a lane); the
// largest magnitudes follow by lane exchanges (and through LDS, where several waves share a page), and with them the scale: the least
// power of two that leaves nothing above 448 = 0.875 * 2^9, taken from the exponent and the mantissa of the largest magnitude.  The same
// registers give the page's score (Alg. 1: the mean of the tokens' norm ratios, as score_blocks.hip has it), so that an eviction does not need
// the page in full precision again.
//
// Bound by memory: a page is read once and half (fp32: a quarter) of it written.  256 rows of D = 128 x 2048 in bfloat16, 402 MB, take 70 us (5.7 TB/s)
// where the caches hold a part of them; else 72 to 77 with pages in order and 84 with shuffled ones, of which 2 KiB are written at a time (a copy of
// as many bytes takes 77).  Stores with the non-temporal hint too, shuffled: 78 and 79 to 81; without it on the loads 65 and 84, on neither 84 and 85.
#include "pe_device.h"
#include "pe_norms.h"
#include "pe_quant.h"
#include "pe_rope_device.h"

namespace pe {
namespace {

// The scale's exponent for a largest magnitude.  448 * 2^e: mantissa 1.75, exponent 8 + e.  (A magnitude below the normal numbers
// counts as the least of them: the scale is 2^-126 at least.)
__device__ __forceinline__ int scale_exponent(float most) {
  const uint32_t u = __float_as_uint(most);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  if (e < -126) e = -126;
  return most == 0.f ? 0 : e;
}
// 2^e, e from -127 + 1 to 127
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// A 16-byte vector's largest magnitude, and its elements times `inv`, rounded to e4m3 (to nearest, ties to even).
template <typename T>
__device__ __forceinline__ float vec_most(const uint4& v) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < Elem<T>::kPerVec; ++e) m = fmaxf(m, fabsf(vec_elem<T>(v, e)));
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t four_e4m3(const uint4& v, int first, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(vec_elem<T>(v, first) * inv, vec_elem<T>(v, first + 1) * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(vec_elem<T>(v, first + 2) * inv, vec_elem<T>(v, first + 3) * inv, w, true);
  return (uint32_t)w;
}
// `to`: byte address of the vector's first element
template <typename T>
__device__ __forceinline__ void store_e4m3(void* to, const uint4& v, float inv) {
  if constexpr (sizeof(T) == 4) {
    *static_cast<uint32_t*>(to) = four_e4m3<T>(v, 0, inv);
  } else {
    *static_cast<uint2*>(to) = make_uint2(four_e4m3<T>(v, 0, inv), four_e4m3<T>(v, 4, inv));
  }
}

template <int M>
__device__ __forceinline__ float wave_max_step(float v) { return fmaxf(v, lane_xor_f32<M>(v)); }
__device__ __forceinline__ float wave_max(float v) {
  return rows_max(wave_max_step<8>(wave_max_step<4>(wave_max_step<2>(wave_max_step<1>(v)))));
}

constexpr int smaller(int a, int b) { return a < b ? a : b; }

// How a page of one head lies in the lanes of kWaves waves.
template <typename T, int D, int B>
struct Page {
  using G = RowGeom<T, D>;
  static constexpr int LPR = G::kLanesPerRow, TPL = G::kTokensPerLoad;
  static constexpr int kAll = B / TPL;                                     // wave-loads of K
  static constexpr int kLoads = smaller(kAll, smaller(8, LPR / 2));        // of a wave
  static constexpr int kWaves = kAll / kLoads;                             // that share a page
  static constexpr int kTokens = kLoads * TPL;                             // of a wave
  static_assert(kWaves * kLoads == kAll, "whole waves");
};
// What a wave does with its part of a page: k[i], v[i] hold the lane's 16 bytes of token (part) * kTokens + i * TPL + lane / LPR.
template <typename T, int D, int B, typename P>
struct Part {
  static constexpr int kLoads = P::kLoads;

  static __device__ __forceinline__ void most(const uint4 (&k)[kLoads], const uint4 (&v)[kLoads], float& mk, float& mv) {
    mk = mv = 0.f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      mk = fmaxf(mk, vec_most<T>(k[i]));
      mv = fmaxf(mv, vec_most<T>(v[i]));
    }
    mk = wave_max(mk);
    mv = wave_max(mv);
  }

  // The tokens' norm ratios, to[token of the page].
  static __device__ __forceinline__ void ratios(const uint4 (&k)[kLoads], const uint4 (&v)[kLoads], int part, double* to) {
    const int lane = lane_id();
    double sums[2 * kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      sums[i] = sumsq_vec<T>(k[i], 0.0);
      sums[kLoads + i] = sumsq_vec<T>(v[i], 0.0);
    }
    const double ratio = token_ratio_from_partials<kLoads, P::LPR>(sums, lane);
    // every lane holds one of its token rows' ratios: that of load bit_reverse((lane >> 1) & (kLoads - 1))
    const int i = bit_reverse<ilog2(kLoads)>((lane >> 1) & (kLoads - 1)), in_row = lane % P::LPR;
    if (in_row < 2 * kLoads && (in_row & 1) == 0) to[part * P::kTokens + i * P::TPL + lane / P::LPR] = ratio;
  }

  // page_byte: of the head's first element in the pools; row_bytes: between its consecutive tokens.
  static __device__ __forceinline__ void store(const uint4 (&k)[kLoads], const uint4 (&v)[kLoads], int part, const pe_quant_cache& cache,
                                               int64_t page_byte, int row_bytes, float inv_k, float inv_v) {
    const int lane = lane_id();
    const int64_t lane_byte = page_byte + (int64_t)(part * P::kTokens + lane / P::LPR) * row_bytes + lane % P::LPR * Elem<T>::kPerVec;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t at = lane_byte + (int64_t)i * P::TPL * row_bytes;
      store_e4m3<T>(static_cast<char*>(cache.k) + at, k[i], inv_k);
      store_e4m3<T>(static_cast<char*>(cache.v) + at, v[i], inv_v);
    }
  }

  // The mean of a page's ratios, in slot order, rounded once.
  static __device__ __forceinline__ float score(const double* ratio) {
    double sum = 0.0;
#pragma unroll 16
    for (int t = 0; t < B; ++t) sum += ratio[t];
    return (float)(sum / (double)B);
  }
};

// Workgroups of four waves (eight where a page takes them); page j of a row is its slot (j % PAGES)'s in workgroup j / PAGES.
template <typename T, int D, int B>
struct Groups {
  using P = Page<T, D, B>;
  static constexpr int kWaves = P::kWaves > 4 ? P::kWaves : 4;
  static constexpr int kPages = kWaves / P::kWaves;
};

template <typename T, int D, int B>
__global__ __launch_bounds__((Groups<T, D, B>::kWaves * kWave)) void quant_pages_kernel(const QuantPagesArgs a, int groups_per_row) {
  using P = Page<T, D, B>;
  constexpr int kPages = Groups<T, D, B>::kPages;
  using PT = Part<T, D, B, P>;
  __shared__ float most_of[Groups<T, D, B>::kWaves][2];
  __shared__ double ratio[kPages][B];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int slot = wave / P::kWaves, part_wave = wave % P::kWaves;
  const int row = (int)(blockIdx.x / (unsigned)groups_per_row), s = row / a.num_kv_heads, hk = row - s * a.num_kv_heads;
  const int j = (int)(blockIdx.x - (unsigned)row * (unsigned)groups_per_row) * kPages + slot;
  const int len = a.seq_lens[s];
  const int most = len < 0 ? 0 : len / B, full = most < a.max_blocks ? most : a.max_blocks;
  const int64_t table_row = (int64_t)(a.shared ? s : row) * a.max_blocks;
  const int heads = a.shared ? a.num_kv_heads : 1;          // token rows between a head's consecutive tokens
  const bool has = j < full;
  const int from = has || (j == full && j < a.max_blocks && len > 0 && len % B != 0) ? a.src_table[table_row + j] : -1;
  const int to = has ? a.block_table[table_row + j] : -1;
  if (a.admitted != nullptr && a.admitted[s] == 0) return;  // (the workgroup has no other row; behind the loads, which do not wait for it)
  const bool real = has && from >= 0 && to >= 0;
  const int64_t head_row = a.shared ? hk : 0;
  // (16-byte vectors; without a page the pool's first: any address inside will do)
  const int64_t base = from >= 0 ? ((int64_t)from * B * heads + head_row) * P::LPR : 0;
  const uint4* kp = static_cast<const uint4*>(a.k_pool);
  const uint4* vp = static_cast<const uint4*>(a.v_pool);
  if (has) {
    const int64_t lane_vec = base + (int64_t)(part_wave * P::kTokens + lane / P::LPR) * heads * P::LPR + lane % P::LPR;
    uint4 k[P::kLoads], v[P::kLoads];
#pragma unroll
    for (int i = 0; i < P::kLoads; ++i) k[i] = load_vec_stream(kp, real ? lane_vec + (int64_t)i * P::TPL * heads * P::LPR : 0);
#pragma unroll
    for (int i = 0; i < P::kLoads; ++i) v[i] = load_vec_stream(vp, real ? lane_vec + (int64_t)i * P::TPL * heads * P::LPR : 0);
    float mk, mv;
    PT::most(k, v, mk, mv);
    if (P::kWaves > 1 && lane == 0) most_of[wave][0] = mk, most_of[wave][1] = mv;
    if (a.scores != nullptr) PT::ratios(k, v, part_wave, ratio[slot]);
    __syncthreads();  // (as in the other branch: every wave of the workgroup reaches one)
    if constexpr (P::kWaves > 1) {
#pragma unroll
      for (int w = 0; w < P::kWaves; ++w) {
        mk = fmaxf(mk, most_of[slot * P::kWaves + w][0]);
        mv = fmaxf(mv, most_of[slot * P::kWaves + w][1]);
      }
    }
    if (real) {
      const int ek = scale_exponent(mk), ev = scale_exponent(mv);
      PT::store(k, v, part_wave, a.cache, ((int64_t)to * B * heads + head_row) * D, heads * D, exp2i(-ek), exp2i(-ev));
      if (part_wave == 0 && lane == 0) {
        *reinterpret_cast<float2*>(a.cache.scales + ((int64_t)to * heads + head_row) * 2) = make_float2(exp2i(ek), exp2i(ev));
        if (a.scores != nullptr) a.scores[(int64_t)row * a.max_blocks + j] = PT::score(ratio[slot]);
      }
    }
    if (!real && a.scores != nullptr && part_wave == 0 && lane == 0) a.scores[(int64_t)row * a.max_blocks + j] = __builtin_inff();
  } else {
    __syncthreads();
    if (j < a.max_blocks && a.scores != nullptr && part_wave == 0 && lane == 0) a.scores[(int64_t)row * a.max_blocks + j] = __builtin_inff();
    if (from >= 0) {  // the unfinished page
      const int tokens = len - full * B;
      uint4* kt = static_cast<uint4*>(a.cache.k_tail) + (int64_t)row * B * P::LPR;
      uint4* vt = static_cast<uint4*>(a.cache.v_tail) + (int64_t)row * B * P::LPR;
      for (int i = part_wave * kWave + lane; i < tokens * P::LPR; i += P::kWaves * kWave) {
        const int64_t at = base + (int64_t)(i / P::LPR) * heads * P::LPR + i % P::LPR;
        kt[i] = kp[at];
        vt[i] = vp[at];
      }
    }
  }
}

template <typename T, int D, int B>
hipError_t launch_pages(const QuantPagesArgs& a, hipStream_t stream) {
  using G = Groups<T, D, B>;
  const int groups = (a.max_blocks + G::kPages - 1) / G::kPages;
  const int64_t all = (int64_t)a.num_seqs * a.num_kv_heads * groups;
  if (all > ((1LL << 32) - 1) / (G::kWaves * kWave)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((quant_pages_kernel<T, D, B>), dim3((unsigned)all), dim3(G::kWaves * kWave), 0, stream, a, groups);
  return hipGetLastError();
}

struct AppendRope {
  int pairs;  // R / 2; 0: nothing is turned
  int interleaved;
  float magnitude;
  uint64_t turns[64];
};

// N neighbouring elements as fp32, and back (to nearest, ties to even).
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
template <int N>
__device__ __forceinline__ void get(const float* p, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = p[i];
}
template <int N>
__device__ __forceinline__ void get(const bf16_t* p, float (&x)[N]) {
  if constexpr (N == 2) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
    x[0] = bf16_lo_to_f32(w), x[1] = bf16_hi_to_f32(w);
  } else {
    x[0] = __uint_as_float((uint32_t)p->bits << 16);
  }
}
template <int N>
__device__ __forceinline__ void put(float* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = x[i];
}
template <int N>
__device__ __forceinline__ void put(bf16_t* p, const float (&x)[N]) {
  const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[0], x[N - 1]}), bf16x2_t));
  if constexpr (N == 2)
    *reinterpret_cast<uint32_t*>(p) = w;
  else
    p->bits = (uint16_t)w;
}

// As many waves a row as hold a page (up to eight wave-loads of K and of V each); rows of one wave are four to a workgroup.  A lane turns N
// pairs (two, where their number is even) of some of the row's heads, and takes its part of the value; the new token's rows meet in LDS, from
// where they go to the tail, and where they fill the page join the rest of it, which is asked for as soon as the length is there.
//
// Bound: by the chain of a launch (64 rows 3.1 us; 174 rows of D = 128 that all fill, bfloat16, B = 16, 5.6, fp32, B = 128, 9.8); for many rows
// by instructions (8192 rows of D = 128, none filling, 7.4, a sixteenth 10.5, all 23.7).  Pages taken in smaller parts one after the other, each
// waiting for memory, leave more registers and take 6.8, 34 and 29.4 us where all fill.
template <typename T, int D, int B>
struct RowWaves {
  using P = Page<T, D, B>;
  static constexpr int kWaves = P::kWaves;                  // of a row
  static constexpr int kRows = kWaves == 1 ? 4 : 1;         // of a workgroup
  static constexpr int kThreads = kWaves * kRows * kWave;
};

template <typename T, int D, int B, int N>
__global__ __launch_bounds__((RowWaves<T, D, B>::kThreads)) void quant_append_kernel(const QuantAppendArgs a, const AppendRope rope) {
  using P = Page<T, D, B>;
  using PT = Part<T, D, B, P>;
  using RW = RowWaves<T, D, B>;
  constexpr int kUnits = D / (2 * N), kAtOnce = RW::kWaves * kWave / kUnits;  // lanes of a head, heads that a row's waves take at once
  __shared__ __attribute__((aligned(16))) T sm_now[RW::kRows][2][D];
  __shared__ double sm_ratio[RW::kRows][B];
  __shared__ float2 sm_most[RW::kWaves];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int part = RW::kWaves == 1 ? 0 : wave, slot_of_row = RW::kWaves == 1 ? wave : 0;
  const int me = part * kWave + lane;  // in the row
  const int row = (int)blockIdx.x * RW::kRows + slot_of_row;
  if (row >= a.num_seqs * a.num_kv_heads) return;  // (of a row of several waves all or none)
  const int s = row / a.num_kv_heads, hk = row - s * a.num_kv_heads;
  T(*now)[D] = sm_now[slot_of_row];
  const auto row_sync = [] {
    if constexpr (RW::kWaves == 1)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wave's accesses to LDS are carried out in order)
    else
      __syncthreads();
  };
  const int len = a.seq_lens[s];
  const int64_t table_row = a.shared ? s : row;
  const int G = a.num_q_heads / a.num_kv_heads;
  // this lane's elements of a head: N from ea on and N from eb on
  const int p = N * (me & (kUnits - 1));
  const bool turned = p < rope.pairs, apart = turned && !rope.interleaved;
  const int ea = apart ? p : 2 * p, eb = apart ? p + rope.pairs : 2 * p + N;
  // the row's key, its value, then its queries (where they are turned)
  const int heads = 2 + (rope.pairs > 0 ? G : 0);
  constexpr int kSteps = (2 + 8 + kAtOnce - 1) / kAtOnce;
  float x[kSteps][N], y[kSteps][N];
  const int64_t q0 = ((int64_t)s * a.num_q_heads + (int64_t)hk * G) * D;
  const auto base_of = [&](int h) -> const T* {
    return h == 0 ? static_cast<const T*>(a.new_k) + (int64_t)row * D : h == 1 ? static_cast<const T*>(a.new_v) + (int64_t)row * D
                                                                              : static_cast<const T*>(a.q) + q0 + (int64_t)(h - 2) * D;
  };
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int h = i * kAtOnce + me / kUnits;
    if (h < heads) {
      const T* from = base_of(h);
      get(from + ea, x[i]);
      get(from + eb, y[i]);
    }
  }
  Turn w[N];
  if (turned) {
    const int position = a.positions[s];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      w[n] = turn_of(rope.turns[p + n], position);
      w[n].c *= rope.magnitude;
      w[n].s *= rope.magnitude;
    }
  }
  const int slot = len & (B - 1), jb = len / B;
  const bool runs = len >= 0 && jb < a.max_blocks, fills = runs && slot == B - 1;
  int32_t* entry = a.block_table + table_row * a.max_blocks + jb;
  uint4* kt = static_cast<uint4*>(a.cache.k_tail) + (int64_t)row * B * P::LPR;
  uint4* vt = static_cast<uint4*>(a.cache.v_tail) + (int64_t)row * B * P::LPR;
  // a page that fills: its tokens so far (the place of the last one holds something older)
  int page = -1;
  uint4 k[P::kLoads], v[P::kLoads];
  if (fills) {
    page = *entry;
#pragma unroll
    for (int i = 0; i < P::kLoads; ++i) {
      const int at = (part * P::kTokens + i * P::TPL) * P::LPR + lane;
      k[i] = kt[at];
      v[i] = vt[at];
    }
  }
  const auto turn = [](const Turn& t, float& u, float& v) {
    const float u0 = u;
    u = u0 * t.c - v * t.s;
    v = v * t.c + u0 * t.s;
  };
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int h = i * kAtOnce + me / kUnits;
    if (h >= heads) continue;
    if (turned && h != 1) {
      if (N == 1 || apart) {
#pragma unroll
        for (int n = 0; n < N; ++n) turn(w[n], x[i][n], y[i][n]);
      } else {
        turn(w[0], x[i][0], x[i][N - 1]);
        turn(w[N - 1], y[i][0], y[i][N - 1]);
      }
    }
    T* to = h < 2 ? now[h] : static_cast<T*>(a.q_out) + q0 + (int64_t)(h - 2) * D;
    put(to + ea, x[i]);
    put(to + eb, y[i]);
  }
  row_sync();

  if (hk == 0 && me == 0) a.seq_lens_out[s] = runs ? len + 1 : len;
  if (!runs) return;
  if (slot == 0 && me == 0 && (!a.shared || hk == 0)) {
    int link = a.freed_phys[table_row];
    if (link >= 0) {
      a.freed_phys[table_row] = -1;
    } else {
      const int used = a.spare_used[table_row];
      link = used >= 0 && used < a.n_spare ? a.spare[table_row * a.n_spare + used] : -1;
      a.spare_used[table_row] = used + 1;
    }
    *entry = link;
  }
  if (part == 0 && lane < 2 * P::LPR) {
    const int kv = lane / P::LPR, u = lane % P::LPR;
    (kv ? vt : kt)[slot * P::LPR + u] = reinterpret_cast<const uint4*>(now[kv])[u];
  }
  if (!fills) return;
  if (part * P::kTokens + (P::kLoads - 1) * P::TPL + lane / P::LPR == B - 1) {  // the new token, the last of the page
    k[P::kLoads - 1] = reinterpret_cast<const uint4*>(now[0])[lane % P::LPR];
    v[P::kLoads - 1] = reinterpret_cast<const uint4*>(now[1])[lane % P::LPR];
  }
  float mk, mv;
  PT::most(k, v, mk, mv);
  if (a.scores != nullptr) PT::ratios(k, v, part, sm_ratio[slot_of_row]);
  if (RW::kWaves > 1 && lane == 0) sm_most[part] = make_float2(mk, mv);
  row_sync();
  if constexpr (RW::kWaves > 1) {
#pragma unroll
    for (int i = 0; i < RW::kWaves; ++i) mk = fmaxf(mk, sm_most[i].x), mv = fmaxf(mv, sm_most[i].y);
  }
  if (page < 0) return;  // spare list exhausted (precondition violated): the page is dropped
  const int rows = a.shared ? a.num_kv_heads : 1, head_row = a.shared ? hk : 0;
  const int ek = scale_exponent(mk), ev = scale_exponent(mv);
  PT::store(k, v, part, a.cache, ((int64_t)page * B * rows + head_row) * D, rows * D, exp2i(-ek), exp2i(-ev));
  if (me == 0) {
    *reinterpret_cast<float2*>(a.cache.scales + ((int64_t)page * rows + head_row) * 2) = make_float2(exp2i(ek), exp2i(ev));
    if (a.scores != nullptr) a.scores[(int64_t)row * a.max_blocks + jb] = PT::score(sm_ratio[slot_of_row]);
  }
}

template <typename T, int D, int B>
hipError_t launch_append(const QuantAppendArgs& a, const AppendRope& rope, hipStream_t stream) {
  using RW = RowWaves<T, D, B>;
  const unsigned groups = (unsigned)((a.num_seqs * a.num_kv_heads + RW::kRows - 1) / RW::kRows);
  const auto kernel = rope.pairs % 2 == 0 ? quant_append_kernel<T, D, B, 2> : quant_append_kernel<T, D, B, 1>;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(RW::kThreads), 0, stream, a, rope);
  return hipGetLastError();
}

// f(type, head size, page size) as template arguments
template <typename T, int D, typename F>
hipError_t with_block(int block_size, F f) {
  switch (block_size) {
    case 16: return f.template operator()<T, D, 16>();
    case 32: return f.template operator()<T, D, 32>();
    case 64: return f.template operator()<T, D, 64>();
    case 128: return f.template operator()<T, D, 128>();
    default: return hipErrorInvalidValue;
  }
}
template <typename F>
hipError_t with_shape(bool is_bf16, int head_dim, int block_size, F f) {
  if (head_dim == 64) return is_bf16 ? with_block<bf16_t, 64>(block_size, f) : with_block<float, 64>(block_size, f);
  if (head_dim == 128) return is_bf16 ? with_block<bf16_t, 128>(block_size, f) : with_block<float, 128>(block_size, f);
  return hipErrorInvalidValue;
}
struct PagesLaunch {
  const QuantPagesArgs& a;
  hipStream_t stream;
  template <typename T, int D, int B>
  hipError_t operator()() const { return launch_pages<T, D, B>(a, stream); }
};
struct AppendLaunch {
  const QuantAppendArgs& a;
  const AppendRope& rope;
  hipStream_t stream;
  template <typename T, int D, int B>
  hipError_t operator()() const { return launch_append<T, D, B>(a, rope, stream); }
};

}  // namespace

bool quant_pages_launches(const pe_cache_desc* d) {
  // (a page a workgroup of 512 threads at most)
  return (int64_t)d->num_seqs * d->num_kv_heads * d->max_blocks <= ((1LL << 32) - 1) / 512;
}

hipError_t launch_quant_pages(const QuantPagesArgs& a, hipStream_t stream) {
  return with_shape(a.is_bf16, a.head_dim, a.block_size, PagesLaunch{a, stream});
}

hipError_t launch_quant_append(const QuantAppendArgs& a, const pe_rope* rope, hipStream_t stream) {
  AppendRope r{};
  if (rope != nullptr) {
    r.pairs = rope->rotary_dim / 2;
    r.interleaved = rope->pairs == PE_ROPE_INTERLEAVED;
    r.magnitude = rope->magnitude;
    for (int i = 0; i < 64; ++i) r.turns[i] = rope->turns[i];
  }
  return with_shape(a.is_bf16, a.head_dim, a.block_size, AppendLaunch{a, r, stream});
}

}  // namespace pe
