// Host-side checks that the files of the C-ABI layer share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "../../include/pe.h"

namespace pe {
namespace host {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The decode workgroup shapes that a descriptor may name.
inline bool decode_shape_built(int shape) { return shape == 422 || shape == 424 || shape == 432 || shape == 822; }

// PE_OK if the descriptor names a shape the kernels are built for.
inline int check_desc(const pe_cache_desc* d) {
  if (d == nullptr) return PE_ERR_INVALID_ARG;
  if (d->dtype != PE_F32 && d->dtype != PE_BF16) return PE_ERR_UNSUPPORTED;
  if (d->num_seqs < 1 || d->num_kv_heads < 1 || d->num_q_heads < 1 || d->max_blocks < 1 || d->num_phys_blocks < 1)
    return PE_ERR_INVALID_ARG;
  if (d->num_q_heads % d->num_kv_heads != 0) return PE_ERR_INVALID_ARG;
  if (d->num_q_heads / d->num_kv_heads > 8) return PE_ERR_UNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 128) return PE_ERR_UNSUPPORTED;
  if (d->block_size != 16 && d->block_size != 32 && d->block_size != 64 && d->block_size != 128)
    return PE_ERR_UNSUPPORTED;
  if (d->layout != PE_LAYOUT_PER_HEAD && d->layout != PE_LAYOUT_SHARED) return PE_ERR_UNSUPPORTED;
  if (d->num_phys_blocks > 0x7fffffffLL) return PE_ERR_UNSUPPORTED;
  if ((int64_t)d->num_seqs * d->num_kv_heads > 0x7fffffffLL / 64) return PE_ERR_UNSUPPORTED;
  if (d->decode_splits < 0 || d->decode_splits > 256) return PE_ERR_INVALID_ARG;
  if (d->decode_flat_order != 0 && d->decode_flat_order != 1) return PE_ERR_INVALID_ARG;
  if (d->decode_shape != 0) {
    if (!decode_shape_built(d->decode_shape)) return PE_ERR_UNSUPPORTED;
    const bool tunable = d->dtype == PE_BF16 && d->head_dim == 128 && d->num_q_heads / d->num_kv_heads == 4 &&
                         d->layout == PE_LAYOUT_PER_HEAD;
    if (d->decode_shape != 422 && !tunable) return PE_ERR_UNSUPPORTED;
  }
  return PE_OK;
}

// Compute units of the current device, asked of the HIP runtime once per device.  Without a device (or on an
// error) the count of an MI355X is assumed; the sticky error state of the runtime is left clean.
inline int compute_units() {
  constexpr int kMaxDevices = 64, kDefault = 256;
  static std::atomic<int> cached[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)hipGetLastError();
    return kDefault;
  }
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
    (void)hipGetLastError();
    return kDefault;
  }
  cached[dev].store(n, std::memory_order_relaxed);
  return n;
}

uint64_t launch_tag();  // of a launch whose splits are merged by the last to arrive (pe_api.hip)

// A row of workgroups has fewer than 2^32 threads.
inline bool one_launch(int64_t workgroups, int threads) { return workgroups <= ((1LL << 32) - 1) / threads; }

inline int check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return PE_OK;
  if (ws == nullptr || have < need || !aligned(ws, 256)) return PE_ERR_WORKSPACE;
  return PE_OK;
}

// A structure that pe_rope_init has filled, for heads of this size.
inline bool rope_ok(const pe_rope* r, int head_dim) {
  return r != nullptr && r->filled == 1 && r->rotary_dim >= 2 && r->rotary_dim <= head_dim && r->rotary_dim % 2 == 0 &&
         (r->pairs == PE_ROPE_HALF || r->pairs == PE_ROPE_INTERLEAVED);
}

inline bool finite(float x) { return x == x && x - x == 0.f; }

inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

}  // namespace host
}  // namespace pe
