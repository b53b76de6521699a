// Pages of a cache rounded to e4m3 (pe_quant_pages), and a decode step's new token, with the page that it fills (pe_quant_append).
//
// A page of a head is read once into registers, by as many waves as hold it (kLoads 16-byte loads of K and of V a lane); the
// largest magnitudes follow by lane exchanges (and through LDS, where several waves share a page), and with them the scale: the least
// power of two that leaves nothing above 448 = 0.875 * 2^9, taken from the exponent and the mantissa of the largest magnitude.  The same
// registers give the page's score (Alg. 1: the mean of the tokens' norm ratios, as score_blocks.hip has it), so that an eviction does not need
// the page in full precision again.
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
constexpr int kMostWaves = 8;

// What the waves of a workgroup leave for one another.
template <int B, int PAGES>
struct Shared {
  float most[kMostWaves][2];
  double ratio[PAGES][B];
};

// A page in registers: k[i], v[i] hold the lane's 16 bytes of token (wave in page) * kTokens + i * TPL + lane / LPR.  All waves of the workgroup
// call this together (`real`: the wave has a page).  to: the page's number in the cache; part: the head's first byte in the page; row_bytes:
// bytes between a head's consecutive tokens.
template <typename T, int D, int B, int PAGES>
__device__ __forceinline__ void round_page(const uint4 (&k)[Page<T, D, B>::kLoads], const uint4 (&v)[Page<T, D, B>::kLoads], bool real, int slot,
                                           int part_wave, Shared<B, PAGES>& sm, const pe_quant_cache& cache, int64_t page_byte, int row_bytes,
                                           int64_t scale_at, float* score) {
  using P = Page<T, D, B>;
  constexpr int N = Elem<T>::kPerVec;
  const int lane = lane_id();
  float mk = 0.f, mv = 0.f;
#pragma unroll
  for (int i = 0; i < P::kLoads; ++i) {
    mk = fmaxf(mk, vec_most<T>(k[i]));
    mv = fmaxf(mv, vec_most<T>(v[i]));
  }
  mk = wave_max(mk);
  mv = wave_max(mv);
  if constexpr (P::kWaves > 1) {
    const int wave = slot * P::kWaves + part_wave;
    if (lane == 0) sm.most[wave][0] = mk, sm.most[wave][1] = mv;
  }
  if (score != nullptr) {
    double part[2 * P::kLoads];
#pragma unroll
    for (int i = 0; i < P::kLoads; ++i) {
      part[i] = sumsq_vec<T>(k[i], 0.0);
      part[P::kLoads + i] = sumsq_vec<T>(v[i], 0.0);
    }
    const double ratio = token_ratio_from_partials<P::kLoads, P::LPR>(part, lane);
    // every lane holds one of its token rows' ratios: load bit_reverse((lane >> 1) & (kLoads - 1))
    const int i = bit_reverse<ilog2(P::kLoads)>((lane >> 1) & (P::kLoads - 1));
    const int in_row = lane % P::LPR;
    if (in_row < 2 * P::kLoads && (in_row & 1) == 0) sm.ratio[slot][part_wave * P::kTokens + i * P::TPL + lane / P::LPR] = ratio;
  }
  __syncthreads();
  if constexpr (P::kWaves > 1) {
#pragma unroll
    for (int w = 0; w < P::kWaves; ++w) {
      mk = fmaxf(mk, sm.most[slot * P::kWaves + w][0]);
      mv = fmaxf(mv, sm.most[slot * P::kWaves + w][1]);
    }
  }
  if (!real) return;
  const int ek = scale_exponent(mk), ev = scale_exponent(mv);
  const float ik = exp2i(-ek), iv = exp2i(-ev);
  const int64_t lane_byte = page_byte + (int64_t)(part_wave * P::kTokens + lane / P::LPR) * row_bytes + lane % P::LPR * N;
#pragma unroll
  for (int i = 0; i < P::kLoads; ++i) {
    const int64_t at = lane_byte + (int64_t)i * P::TPL * row_bytes;
    store_e4m3<T>(static_cast<char*>(cache.k) + at, k[i], ik);
    store_e4m3<T>(static_cast<char*>(cache.v) + at, v[i], iv);
  }
  if (part_wave == 0 && lane == 0) {
    *reinterpret_cast<float2*>(cache.scales + scale_at) = make_float2(exp2i(ek), exp2i(ev));
    if (score != nullptr) {
      double sum = 0.0;
#pragma unroll 16
      for (int t = 0; t < B; ++t) sum += sm.ratio[slot][t];
      *score = (float)(sum / (double)B);
    }
  }
}

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
  constexpr int N = Elem<T>::kPerVec;
  __shared__ Shared<B, kPages> sm;
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
    // (one barrier inside, which all waves of the workgroup reach: here, or in the other branch)
    round_page<T, D, B, kPages>(k, v, real, slot, part_wave, sm, a.cache, ((int64_t)to * B * heads + head_row) * D, heads * D,
                                ((int64_t)to * heads + head_row) * 2, a.scores != nullptr ? a.scores + (int64_t)row * a.max_blocks + j : nullptr);
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

template <typename T>
__device__ __forceinline__ float get(const T* p, int64_t i) {
  if constexpr (sizeof(T) == 4)
    return reinterpret_cast<const float*>(p)[i];
  else
    return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
}
template <typename T>
__device__ __forceinline__ T as(float x) {
  if constexpr (sizeof(T) == 4)
    return x;
  else
    return T{f32_to_bf16(x)};
}

// One workgroup a row: thread i turns pair i % (D/2) of one of the row's query heads, or of the key, and takes its part of the value.  The
// new token meets the rest of its page, where it fills it, in LDS.
template <typename T, int D, int B>
__global__ __launch_bounds__((Groups<T, D, B>::kWaves * kWave)) void quant_append_kernel(const QuantAppendArgs a, const AppendRope rope) {
  using P = Page<T, D, B>;
  constexpr int kThreads = Groups<T, D, B>::kWaves * kWave, kPairs = D / 2;
  __shared__ Shared<B, 1> sm;
  __shared__ __attribute__((aligned(16))) T now[2][D];
  const int me = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(me / kWave);
  const int row = (int)blockIdx.x, s = row / a.num_kv_heads, hk = row - s * a.num_kv_heads;
  const int len = a.seq_lens[s];
  const int slot = len & (B - 1), jb = len / B;
  const bool runs = len >= 0 && jb < a.max_blocks;
  if (hk == 0 && me == 0) a.seq_lens_out[s] = runs ? len + 1 : len;
  const int G = a.num_q_heads / a.num_kv_heads;
  const T* new_k = static_cast<const T*>(a.new_k) + (int64_t)row * D;
  const T* new_v = static_cast<const T*>(a.new_v) + (int64_t)row * D;
  const int p = me & (kPairs - 1);
  const bool turned = p < rope.pairs;
  const int ea = turned && !rope.interleaved ? p : 2 * p, eb = turned && !rope.interleaved ? p + rope.pairs : 2 * p + 1;
  Turn w{1.f, 0.f};
  if (turned) {
    w = turn_of(rope.turns[p], a.positions[s]);
    w.c *= rope.magnitude;
    w.s *= rope.magnitude;
  }
  // heads of the row: its key, its value, then its queries (where they are turned)
  const int heads = 2 + (rope.pairs > 0 ? G : 0);
  for (int h = me / kPairs; h < heads; h += kThreads / kPairs) {
    const int64_t qh = ((int64_t)s * a.num_q_heads + hk * G + (h - 2)) * D;
    const T* from = h == 0 ? new_k : h == 1 ? new_v : static_cast<const T*>(a.q) + qh;
    const float x = get(from, ea), y = get(from, eb);
    const bool turn = turned && h != 1;
    const T u = as<T>(turn ? x * w.c - y * w.s : x), v = as<T>(turn ? y * w.c + x * w.s : y);
    if (h < 2) {
      now[h][ea] = u, now[h][eb] = v;
    } else {
      T* to = static_cast<T*>(a.q_out) + qh;
      to[ea] = u, to[eb] = v;
    }
  }
  __syncthreads();
  if (!runs) return;
  const int64_t table_row = a.shared ? s : row;
  int32_t* entry = a.block_table + table_row * a.max_blocks + jb;
  if (slot == 0 && me == 0 && (!a.shared || hk == 0)) {
    int page = a.freed_phys[table_row];
    if (page >= 0) {
      a.freed_phys[table_row] = -1;
    } else {
      const int used = a.spare_used[table_row];
      page = used >= 0 && used < a.n_spare ? a.spare[table_row * a.n_spare + used] : -1;
      a.spare_used[table_row] = used + 1;
    }
    *entry = page;
  }
  uint4* kt = static_cast<uint4*>(a.cache.k_tail) + (int64_t)row * B * P::LPR;
  uint4* vt = static_cast<uint4*>(a.cache.v_tail) + (int64_t)row * B * P::LPR;
  if (me < 2 * P::LPR) {
    const int kv = me / P::LPR, u = me % P::LPR;
    (kv ? vt : kt)[slot * P::LPR + u] = reinterpret_cast<const uint4*>(now[kv])[u];
  }
  if (slot != B - 1) return;
  // the page is full: its other tokens from the tail, the last one from LDS
  const int page = *entry;
  const bool real = page >= 0 && wave < P::kWaves;
  uint4 k[P::kLoads], v[P::kLoads];
#pragma unroll
  for (int i = 0; i < P::kLoads; ++i) {
    const int t = (real ? wave * P::kTokens : 0) + i * P::TPL + lane / P::LPR, u = lane % P::LPR;
    const bool last = t == B - 1;
    k[i] = last ? reinterpret_cast<const uint4*>(now[0])[u] : kt[t * P::LPR + u];
    v[i] = last ? reinterpret_cast<const uint4*>(now[1])[u] : vt[t * P::LPR + u];
  }
  const int rows = a.shared ? a.num_kv_heads : 1, head_row = a.shared ? hk : 0;
  // (waves beyond those that hold the page take part in the barrier alone)
  if (wave >= P::kWaves) {
    __syncthreads();
    return;
  }
  round_page<T, D, B, 1>(k, v, real, 0, wave, sm, a.cache, ((int64_t)page * B * rows + head_row) * D, rows * D,
                         ((int64_t)page * rows + head_row) * 2, a.scores != nullptr ? a.scores + (int64_t)row * a.max_blocks + jb : nullptr);
}

template <typename T, int D, int B>
hipError_t launch_append(const QuantAppendArgs& a, const AppendRope& rope, hipStream_t stream) {
  hipLaunchKernelGGL((quant_append_kernel<T, D, B>), dim3((unsigned)(a.num_seqs * a.num_kv_heads)), dim3(Groups<T, D, B>::kWaves * kWave), 0,
                     stream, a, rope);
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
