// Rotary positions of queries and keys: every pair of channels turned by an angle proportional to the token's
// position, before the gauge sees the key.
//
// Pair i of a token at position p turns by p f_i radians (f_i falls geometrically with i).  In binary32 p f_i
// is off by whole radians at far positions, so the frequency is held in turns as a 64-bit fraction F = f / 2 pi (within
// 2^-63): p F modulo 2^64 is the angle modulo one turn, to p 2^-63, by two integer products.  The nearest
// quarter turn comes off in integers too; sine and cosine of the rest (at most pi / 4) are Taylor polynomials
// whose first dropped terms are below 2^-28.
//
// A token's angles serve all heads and layers, so a thread keeps the sines and cosines of V pairs of one token
// and walks `per` (layer, head) rows, 16-byte loads where the widths allow.  Bound by memory: every element is
// read and written once.  8192 tokens x 40 heads of 128 channels, bf16: 30.0 us = 5.6 TB/s (an addition in place over
// 1 GiB reaches 6.0).
#include <algorithm>

#include "cg_internal.h"
#include "cg_device.h"
#include "cg_rope.h"

namespace cg {

namespace {

template <int V, bool BF16, int LAYOUT>
__global__ __launch_bounds__(256) void rope_rows(RopeArgs a) {
  constexpr int ES = BF16 ? 2 : 4;
  const int idx = blockIdx.x * 256 + threadIdx.x;
  const int u = idx % a.units, tk = idx / a.units, T = a.x[0].T;
  if (tk >= a.x[0].B * T || u >= a.skip) return;
  const int b = tk / T, t = tk - b * T;
  const int p = a.pos[tk];
  if (p < 0) return;  // padding: the row stays as it was
  const int hr = a.plan.d_rot / 2;
  const bool turn = u < hr / V;
  float sn[V], cn[V];
  if (turn) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sincos_turns(uint64_t(uint32_t(p)) * a.plan.step[u * V + i], sn[i], cn[i]);
      sn[i] *= a.inverse ? -a.plan.amplitude : a.plan.amplitude;
      cn[i] *= a.plan.amplitude;
    }
  }
  // first and second run of V channels of the unit
  const int c0 = LAYOUT == CG_ROPE_HALF && turn ? u * V : 2 * u * V;
  const int c1 = LAYOUT == CG_ROPE_HALF && turn ? hr + u * V : c0 + V;
  const int n0 = a.x[0].L * a.x[0].H, rows = n0 + (a.x[1].H ? a.x[1].L * a.x[1].H : 0);
  const int r1 = min(rows, int(blockIdx.y + 1) * a.per);
#pragma unroll 2
  for (int r = blockIdx.y * a.per; r < r1; ++r) {
    const int k = r >= n0, rr = k ? r - n0 : r;
    const ViewDev &X = a.x[k], &Y = a.y[k];
    const int lv = rr / X.H, h = rr - lv * X.H;
    const char* src = static_cast<const char*>(X.ptr) + ES * (lv * X.sl + b * X.sb + h * X.sh + t * X.st);
    char* dst = static_cast<char*>(Y.ptr) + ES * (lv * Y.sl + b * Y.sb + h * Y.sh + t * Y.st);
    turn_row<V, BF16, LAYOUT>(src, dst, c0, c1, turn, sn, cn);
  }
}

template <int V, bool BF16>
const void* rope_fn(int layout) {
  return layout == CG_ROPE_HALF ? (const void*)rope_rows<V, BF16, CG_ROPE_HALF> : (const void*)rope_rows<V, BF16, CG_ROPE_PAIRS>;
}
template <bool BF16>
const void* rope_by_width(int V, int layout) {
  if constexpr (BF16) {
    if (V == 8) return rope_fn<8, true>(layout);
  }
  return V == 4 ? rope_fn<4, BF16>(layout) : V == 2 ? rope_fn<2, BF16>(layout) : rope_fn<1, BF16>(layout);
}

}  // namespace

bool rope_split(const cg_rope_plan& plan, const ViewDev& x0, const ViewDev& y0, const ViewDev& x1, const ViewDev& y1,
                const int* pos, bool inverse, RopeSplit& s) {
  RopeArgs& a = s.a;
  a.plan = plan;
  a.x[0] = x0; a.x[1] = x1;
  a.y[0] = y0; a.y[1] = y1;
  a.pos = pos;
  a.inverse = inverse;
  const int d = x0.d;
  // pairs a thread takes: the most that rows and rotated part divide into, up to 16 bytes of neighbours (binary32, 2
  // layers x 3 x 1021 tokens x 32 heads of 64 channels: 29.2 us with eight, whose loads lie 64 bytes apart, 24.8 with four)
  int V = x0.bf16 ? 8 : 4;
  while (d % (2 * V) || plan.d_rot % (2 * V)) V /= 2;
  a.units = d / (2 * V);
  auto same = [](const ViewDev& x, const ViewDev& y) {
    return x.ptr == y.ptr && x.sl == y.sl && x.sb == y.sb && x.sh == y.sh && x.st == y.st;
  };
  const bool in_place = same(x0, y0) && (x1.H == 0 || same(x1, y1));
  a.skip = in_place ? plan.d_rot / (2 * V) : a.units;
  const int64_t tokens = int64_t(x0.B) * x0.T;
  const int rows = x0.L * x0.H + (x1.H ? x1.L * x1.H : 0);
  s.V = V;
  s.gx = s.gy = 0;
  if (tokens == 0 || a.skip == 0) return true;
  const int64_t blocks = (tokens * a.units + 255) / 256;
  if (tokens * a.units > 0x7fffff00) return false;
  // rows per thread: as many as leave about four workgroups per CU, at most 8 (8192 tokens x 40 heads: one 41 us, up to
  // four 31.6, eight 30.0, sixteen 30.1; eight workgroups per CU 31.1)
  a.per = int(std::max<int64_t>(1, std::min<int64_t>(8, blocks * rows / (4 * cu_count()))));
  s.gx = unsigned(blocks);
  s.gy = (rows + a.per - 1) / a.per;
  return s.gy <= 65535;
}

hipError_t launch_rope(const cg_rope_plan& plan, const ViewDev& x0, const ViewDev& y0, const ViewDev& x1, const ViewDev& y1,
                       const int* pos, bool inverse, hipStream_t st) {
  RopeSplit s;
  if (!rope_split(plan, x0, y0, x1, y1, pos, inverse, s)) return hipErrorInvalidValue;
  return launch_rope_split(s, st);
}

hipError_t launch_rope_split(const RopeSplit& s, hipStream_t st) {
  if (s.gx == 0) return hipSuccess;
  const int layout = s.a.plan.layout;
  const void* fn = s.a.x[0].bf16 ? rope_by_width<true>(s.V, layout) : rope_by_width<false>(s.V, layout);
  void* args[] = {const_cast<RopeArgs*>(&s.a)};
  return hipLaunchKernel(fn, dim3(s.gx, s.gy), dim3(256), args, 0, st);
}

}  // namespace cg
