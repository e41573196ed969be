// Sine and cosine of rotary positions, shared by the rope kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.h"
#include "rope.hpp"

namespace cp {

// (cos, sin) of pos * f turns, times the magnitude. The product is formed and
// reduced to half a turn in 64 bits (at position 10^6 a 32-bit product is off by
// 0.03 turns); what the 32-bit remainder drops turns the result once more.
CP_DEV float2 rope_turn(const RopeK &r, int64_t pos, int32_t pair) {
  const double x = (double)pos * r.turns[pair];
  const double t = x - rint(x);
  const float th = (float)t, tl = (float)(t - (double)th) * 6.2831853f;
  float s, c;
  sincospif(2.f * th, &s, &c);
  const float c2 = __builtin_fmaf(-tl, s, c), s2 = __builtin_fmaf(tl, c, s);
  return float2{c2 * r.magnitude, (r.inverse ? -s2 : s2) * r.magnitude};
}

// The two elements of a pair, turned by t = (cos, sin).
CP_DEV float rope_first(float a, float b, float2 t) { return __builtin_fmaf(a, t.x, -(b * t.y)); }
CP_DEV float rope_second(float a, float b, float2 t) { return __builtin_fmaf(a, t.y, b * t.x); }

}  // namespace cp
