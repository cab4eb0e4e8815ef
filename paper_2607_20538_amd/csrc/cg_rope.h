// Sine and cosine of a rotation's angles (one copy per translation unit; the angles: cg_rope.hip).
#pragma once

#include "cg_internal.h"

namespace cg {
namespace {

// turns (64-bit fraction) -> sine and cosine
__device__ __forceinline__ void sincos_turns(uint64_t f, float& s, float& c) {
  const uint32_t q = uint32_t((f + (uint64_t(1) << 61)) >> 62);
  const int64_t r = int64_t(f - (uint64_t(q) << 62));  // within an eighth of a turn
  const float x = float(int32_t(r >> 32)) * 1.46291807926715968e-9f;  // 2 pi 2^-32
  const float x2 = x * x;
  float a = fmaf(x2, 2.755731922398589e-6f, -1.984126984126984e-4f);  // 1/9!, -1/7!
  a = fmaf(x2, a, 8.333333333333333e-3f);
  a = fmaf(x2, a, -1.666666666666667e-1f);
  a = fmaf(x * x2, a, x);
  float b = fmaf(x2, -2.755731922398589e-7f, 2.480158730158730e-5f);  // -1/10!, 1/8!
  b = fmaf(x2, b, -1.388888888888889e-3f);
  b = fmaf(x2, b, 4.166666666666667e-2f);
  b = fmaf(x2, b, -0.5f);
  b = fmaf(x2, b, 1.0f);
  s = (q & 1) ? b : a;
  c = (q & 1) ? a : b;
  if (q & 2) s = -s;
  if ((q + 1) & 2) c = -c;
}

// What turns a pair at position p >= 0: amplitude times sine and cosine
__device__ __forceinline__ void pair_turn(const cg_rope_plan& plan, int pair, int p, float& s, float& c) {
  sincos_turns(uint64_t(uint32_t(p)) * plan.step[pair], s, c);
  s *= plan.amplitude;
  c *= plan.amplitude;
}
__device__ __forceinline__ void turn_pair(float& x0, float& x1, float s, float c) {
  const float y0 = fmaf(x0, c, -(x1 * s));
  x1 = fmaf(x0, s, x1 * c);
  x0 = y0;
}
// Channels of a pair
__device__ __forceinline__ void pair_channels(const cg_rope_plan& plan, int pair, int& c0, int& c1) {
  const bool half = plan.layout == CG_ROPE_HALF;
  c0 = half ? pair : 2 * pair;
  c1 = half ? pair + plan.d_rot / 2 : c0 + 1;
}

}  // namespace
}  // namespace cg
