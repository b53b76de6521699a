// Rotary positions of queries and keys, and the turned keys' and the values' way into the pages (pe_rotate).
//
// Bound by memory: every element is read and written once (stored keys written twice), the angles cost some thirty instructions for
// each pair of a token, whatever the number of heads.  A workgroup takes some tokens: first its threads put the cosines and
// sines of their pairs into LDS, then they walk over (token, head, part), 16 bytes of each half of a pair at a time (neighbouring
// pairs: 16 bytes), the next ones on their way while these are turned.  What is written does not pass through the caches (854 MB moved, with keys
// and values stored: 146 us or 5.9 TB/s, a copy reaches 5.2; with ordinary stores 152; fp32, 36 MB: 6.6 us, 8.2).
//
// Where rows are not 16-byte aligned, or a half is no multiple of 16 bytes, threads walk over single pairs instead, 2 bytes (fp32: 4) an access with
// a division and a look at the slot for each: 32004 tokens of 32 + 8 heads of D = 128, stored, bfloat16, rotary 40 294 us, rotary 128 in rows
// 2 bytes off 292 (2.9 TB/s; 146 by vectors), neighbours as pairs 281 to 288; 8000 tokens of fp32, rotary 40 95 us, rows 4 bytes off 109 (63).
#include "pe_rope_device.h"
#include "pe_tokens.h"

namespace pe {
namespace {

constexpr int kThreads = kRotateThreads;
constexpr int kMostPairs = 64;

// Elements of 16 bytes as fp32, and back.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Vec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = vec_elem<bf16_t>(r, e);
  }
  static __device__ __forceinline__ uint32_t two(float a, float b) {  // to nearest, ties to even
    typedef __attribute__((ext_vector_type(2))) float f32x2_t;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[8]) {
    return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
  }
};

template <typename T>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 4)
    return static_cast<const float*>(p)[i];
  else
    return __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
}
template <typename T>
__device__ __forceinline__ void store_one(void* p, int64_t i, float x) {
  if constexpr (sizeof(T) == 4)
    static_cast<float*>(p)[i] = x;
  else
    static_cast<uint16_t*>(p)[i] = f32_to_bf16(x);
}

// Where head h of the batch's queries, keys and values (numbered in this order) is read and written.
struct Head {
  const void* from;
  void* to;       // null: not kept
  int64_t in, out;  // element of the head's first
  int kv;         // its number among the keys or values, or -1
  bool value;
};
__device__ __forceinline__ Head head_of(const RotateArgs& a, int64_t t, int h) {
  if (h < a.num_q_heads) return Head{a.q, a.q_out, t * a.q_stride + (int64_t)h * a.head_dim, t * a.q_out_stride + (int64_t)h * a.head_dim, -1, false};
  h -= a.num_q_heads;
  if (h < a.num_kv_heads) return Head{a.k, a.k_out, t * a.k_stride + (int64_t)h * a.head_dim, t * a.k_out_stride + (int64_t)h * a.head_dim, h, false};
  h -= a.num_kv_heads;
  return Head{a.v, nullptr, t * a.v_stride + (int64_t)h * a.head_dim, 0, h, true};
}
// The head's first element in the pools, or -1.
__device__ __forceinline__ int64_t pool_at(const RotateArgs& a, int64_t t, const Head& head) {
  if (a.slots == nullptr || head.kv < 0) return -1;
  const int64_t slot = a.shared ? a.slots[t] : a.slots[t * a.num_kv_heads + head.kv];
  if (slot < 0 || slot >= a.pool_tokens) return -1;
  return (a.shared ? slot * a.num_kv_heads + head.kv : slot) * a.head_dim;
}

struct Rope {
  int pairs;  // R / 2
  float magnitude;
  uint64_t turns[kMostPairs];
};

// Cosines and sines of `count` tokens' pairs, times the magnitude.
__device__ __forceinline__ void fill_turns(Turn* sm, const Rope& rope, const int32_t* positions, int64_t t0, int count, bool transpose) {
  for (int i = (int)threadIdx.x; i < count * kMostPairs; i += kThreads) {
    const int t = i / kMostPairs, p = i % kMostPairs;
    if (p >= rope.pairs) continue;
    Turn x = turn_of(rope.turns[p], positions[t0 + t]);
    x.c *= rope.magnitude;
    x.s *= transpose ? -rope.magnitude : rope.magnitude;
    sm[t * kMostPairs + p] = x;
  }
  __syncthreads();
}

// Single pairs (i, i + R/2) or (2i, 2i + 1), and what is behind them two elements at a time.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotate_pairs_kernel(const RotateArgs a, const Rope rope, int heads) {
  __shared__ Turn sm[kMostPairs];
  const int64_t t = blockIdx.x;
  fill_turns(sm, rope, a.positions, t, 1, a.transpose);
  const int half = a.head_dim / 2;
  for (int i = (int)threadIdx.x; i < heads * half; i += kThreads) {
    const int h = i / half, p = i % half;
    const Head head = head_of(a, t, h);
    const int64_t pool = pool_at(a, t, head);
    if (head.value && pool < 0) continue;
    const bool turned = p < rope.pairs;
    const int ea = !turned || INTERLEAVED ? 2 * p : p, eb = !turned || INTERLEAVED ? 2 * p + 1 : p + rope.pairs;
    float x = load_one<T>(head.from, head.in + ea), y = load_one<T>(head.from, head.in + eb);
    if (turned && !head.value) {
      const Turn w = sm[p];
      const float x0 = x;
      x = x0 * w.c - y * w.s;
      y = y * w.c + x0 * w.s;
    }
    // (value heads go by 2p, 2p + 1 or by halves alike: each element is one thread's)
    if (head.to != nullptr) store_one<T>(head.to, head.out + ea, x), store_one<T>(head.to, head.out + eb, y);
    if (pool >= 0) {
      void* to = head.value ? a.v_pool : a.k_pool;
      store_one<T>(to, pool + ea, x), store_one<T>(to, pool + eb, y);
    }
  }
}

// 16 bytes at a time.  A head has `units` of work: of each half 16 bytes (INTERLEAVED: 16 bytes) turned, then 16 bytes copied; of a value
// head twice 16 bytes copied.  The first unit's elements are asked for in front of the angles, the next one's in front of the stores.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a, const Rope rope, int heads, int tokens_each, int log2_units,
                                                          uint32_t inv_heads) {
  constexpr int N = Vec<T>::N;
  extern __shared__ Turn turns[];
  const int64_t t0 = (int64_t)blockIdx.x * tokens_each;
  const int count = a.tokens - t0 < tokens_each ? (int)(a.tokens - t0) : tokens_each;
  const int nturned = INTERLEAVED ? 2 * rope.pairs / N : rope.pairs / N;  // units that turn
  const int nvec = a.head_dim / N;
  const int units = 1 << log2_units, u = (int)threadIdx.x & (units - 1);
  const int all = count * heads;

  struct Unit {
    uint4* to;
    uint4* page;
    int token, first, second;  // its vectors of a head; second -1: one alone
    bool turned;
    uint4 x, y;
  };
  const auto load = [&](int i) {
    Unit w{};
    w.first = w.second = -1;
    if (i >= all) return w;
    const int t = tokens_each == 1 ? 0 : heads == 1 ? i : (int)((uint64_t)(uint32_t)i * inv_heads >> 32), h = i - t * heads;
    const Head head = head_of(a, t0 + t, h);
    const int64_t pool = pool_at(a, t0 + t, head);
    w.token = t;
    w.to = head.to == nullptr ? nullptr : reinterpret_cast<uint4*>(static_cast<T*>(head.to) + head.out);
    w.page = pool < 0 ? nullptr : reinterpret_cast<uint4*>(static_cast<T*>(head.value ? a.v_pool : a.k_pool) + pool);
    if (head.value) {
      if (w.page == nullptr) return w;
      if (u < nvec) w.first = u;
      if (u + units < nvec) w.second = u + units;
    } else if (u < nturned) {
      w.turned = true;
      w.first = u;
      if (!INTERLEAVED) w.second = u + nturned;
    } else if (u + (INTERLEAVED ? 0 : nturned) < nvec) {
      w.first = u + (INTERLEAVED ? 0 : nturned);
    }
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(head.from) + head.in);
    if (w.first >= 0) w.x = from[w.first];
    if (w.second >= 0) w.y = from[w.second];
    return w;
  };
  const auto finish = [&](Unit& w) {
    if (w.turned) {
      const Turn* r = turns + w.token * kMostPairs;
      float x[N], y[N];
      Vec<T>::get(w.x, x);
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          const Turn v = r[u * (N / 2) + e];
          const float p = x[2 * e], q = x[2 * e + 1];
          x[2 * e] = p * v.c - q * v.s;
          x[2 * e + 1] = q * v.c + p * v.s;
        }
      } else {
        Vec<T>::get(w.y, y);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const Turn v = r[u * N + e];
          const float p = x[e], q = y[e];
          x[e] = p * v.c - q * v.s;
          y[e] = q * v.c + p * v.s;
        }
        w.y = Vec<T>::put(y);
      }
      w.x = Vec<T>::put(x);
    }
    if (w.first >= 0) {
      if (w.to != nullptr) store_vec_stream(w.to, w.first, w.x);
      if (w.page != nullptr) store_vec_stream(w.page, w.first, w.x);
    }
    if (w.second >= 0) {
      if (w.to != nullptr) store_vec_stream(w.to, w.second, w.y);
      if (w.page != nullptr) store_vec_stream(w.page, w.second, w.y);
    }
  };

  const int step = kThreads >> log2_units;
  int i = (int)threadIdx.x >> log2_units;
  Unit now = load(i);
  fill_turns(turns, rope, a.positions, t0, count, a.transpose);
  for (; i < all; i += step) {
    Unit next = load(i + step);
    finish(now);
    now = next;
  }
}

template <typename T>
bool by_vectors(const RotateArgs& a, const pe_rope& rope) {
  constexpr int N = Vec<T>::N;
  const auto fits = [](const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % N == 0; };
  return rope.rotary_dim % (rope.pairs == PE_ROPE_INTERLEAVED ? N : 2 * N) == 0 && fits(a.q, a.q_stride) && fits(a.k, a.k_stride) &&
         fits(a.v, a.v_stride) && fits(a.q_out, a.q_out_stride) && fits(a.k_out, a.k_out_stride) && fits(a.k_pool, 0) && fits(a.v_pool, 0);
}

// Tokens of a workgroup: one where it has 5 KiB or more to turn (workgroups that are soon through stream best: 32004 tokens of 32 + 8 heads of D =
// 128 in one | two | four tokens 152 | 163 | 169 us, of D = 64 87 | 95 | 103), as many as that takes of few heads where tokens are many (67000 of 2 + 1
// heads of D = 128 71 | 41 | 30, eight 27; fp32 106 | 81 | 69; 32004 of 8 + 2 39 | 34 | 34; not 500 of these: 4.2 | 4.3 | 5.7).
constexpr int kMostTokens = 8;
int tokens_each(int64_t tokens, int token_bytes) {
  int each = 1;
  while (each < kMostTokens && each * token_bytes < 5 << 10 && tokens >= each * 2048) each *= 2;
  return each;
}

template <typename T, bool INTERLEAVED>
hipError_t launch(const RotateArgs& a, const pe_rope& rope, hipStream_t stream) {
  Rope r;
  r.pairs = rope.rotary_dim / 2;
  r.magnitude = rope.magnitude;
  for (int i = 0; i < kMostPairs; ++i) r.turns[i] = rope.turns[i];
  const int heads = a.num_q_heads + a.num_kv_heads * (a.slots != nullptr ? 2 : 1);
  if (!by_vectors<T>(a, rope)) {
    hipLaunchKernelGGL((rotate_pairs_kernel<T, INTERLEAVED>), dim3((unsigned)a.tokens), dim3(kThreads), 0, stream, a, r, heads);
    return hipGetLastError();
  }
  constexpr int N = Vec<T>::N;
  const int units = a.head_dim / N - (INTERLEAVED ? 0 : r.pairs / N);
  int log2_units = 0;  // (of a value head: half of its vectors at least)
  while ((1 << log2_units) < units) ++log2_units;
  const int each = tokens_each(a.tokens, heads * a.head_dim * (int)sizeof(T));
  const int64_t groups = (a.tokens + each - 1) / each;
  // i / heads is the upper half of i * inv_heads (several tokens: few heads)
  const uint32_t inv_heads = (uint32_t)((1ull << 32) / (uint32_t)heads + 1);
  hipLaunchKernelGGL((rotate_kernel<T, INTERLEAVED>), dim3((unsigned)groups), dim3(kThreads), each * kMostPairs * sizeof(Turn), stream, a, r, heads,
                     each, log2_units, inv_heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& all, const pe_rope& rope, hipStream_t stream) {
  const bool inter = rope.pairs == PE_ROPE_INTERLEAVED;
  const int64_t bytes = all.is_bf16 ? 2 : 4, most = ((1LL << 32) - 1) / kThreads;  // a launch has fewer than 2^32 threads
  const auto behind = [&](const void* p, int64_t elements) {
    return p == nullptr ? static_cast<const char*>(nullptr) : static_cast<const char*>(p) + elements * bytes;
  };
  for (int64_t t = 0; t < all.tokens; t += most) {
    RotateArgs a = all;
    a.tokens = all.tokens - t < most ? all.tokens - t : most;
    a.positions = all.positions + t;
    a.q = behind(all.q, t * all.q_stride);
    a.k = behind(all.k, t * all.k_stride);
    a.v = behind(all.v, t * all.v_stride);
    a.q_out = const_cast<char*>(behind(all.q_out, t * all.q_out_stride));
    a.k_out = const_cast<char*>(behind(all.k_out, t * all.k_out_stride));
    if (a.slots != nullptr) a.slots = all.slots + t * (all.shared ? 1 : all.num_kv_heads);
    const hipError_t e = a.is_bf16 ? (inter ? launch<bf16_t, true>(a, rope, stream) : launch<bf16_t, false>(a, rope, stream))
                                   : (inter ? launch<float, true>(a, rope, stream) : launch<float, false>(a, rope, stream));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pe
