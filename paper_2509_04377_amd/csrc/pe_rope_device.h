// Cosine and sine of a rotary angle.
#pragma once

#include <stdint.h>

#include "pe_device.h"

namespace pe {

struct Turn {
  float c, s;
};

// position * turns (units of 2^-64 turns) modulo a turn is what the product of 64-bit integers keeps, at any position, negative ones
// too.  The nearest quarter turn is its two upper bits; what is left, within an eighth of a turn, goes through the power
// series of sine and cosine, whose first terms left out are below 2^-28 and 2^-33 there.  (The upper 32 bits of what is left: an angle is off by
// 2^-32 turns at most.)
__device__ __forceinline__ Turn turn_of(uint64_t turns, int32_t position) {
  const uint64_t a = turns * (uint64_t)(int64_t)position + (1ull << 61);
  const uint32_t top = (uint32_t)(a >> 32);
  const uint32_t quarter = top >> 30;
  const float x = (float)((int32_t)(top & 0x3fffffffu) - (1 << 29)) * 1.46291807926715968e-09f;  // 2 pi / 2^32
  const float y = x * x;
  float s = 2.7557319224e-06f;  // 1 / 9!
  s = fmaf(s, y, -1.9841269841e-04f);
  s = fmaf(s, y, 8.3333333333e-03f);
  s = fmaf(s, y, -1.6666666667e-01f);
  s = fmaf(s * y, x, x);
  float c = -2.7557319224e-07f;  // 1 / 10!
  c = fmaf(c, y, 2.4801587302e-05f);
  c = fmaf(c, y, -1.3888888889e-03f);
  c = fmaf(c, y, 4.1666666667e-02f);
  c = fmaf(c, y, -0.5f);
  c = fmaf(c, y, 1.f);
  // (cos, sin) a quarter turn further is (-sin, cos)
  const bool odd = (quarter & 1u) != 0u;
  Turn t{odd ? s : c, odd ? c : s};
  if (quarter == 1u || quarter == 2u) t.c = -t.c;
  if (quarter >= 2u) t.s = -t.s;
  return t;
}

}  // namespace pe
