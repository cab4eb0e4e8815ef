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

struct RopeArgs {
  cg_rope_plan plan;
  ViewDev x[2], y[2];   // queries and keys (the second may be absent: H = 0)
  const int* pos;       // [B][T]
  int inverse, per;     // rows (layer, head) of a thread
  int units, skip;      // units of 2 V channels a row has; units from `skip` on are left (in-place: nothing to copy)
};

// V neighbouring elements, as loaded and as binary32
template <int V, bool BF16>
struct Elems {
  static constexpr int bytes = V * (BF16 ? 2 : 4);
  typedef uint32_t word_t __attribute__((ext_vector_type(bytes >= 16 ? 4 : (bytes >= 8 ? 2 : 1))));
  static constexpr int N = bytes / int(sizeof(word_t)) > 0 ? bytes / int(sizeof(word_t)) : 1;
  word_t w[N];
  __device__ __forceinline__ void load(const char* p) {
    if constexpr (bytes == 2) w[0] = word_t(*reinterpret_cast<const uint16_t*>(p));
    else {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const word_t*>(p + i * sizeof(word_t));
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    if constexpr (bytes == 2) *reinterpret_cast<uint16_t*>(p) = uint16_t(w[0][0]);
    else {
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<word_t*>(p + i * sizeof(word_t)) = w[i];
    }
  }
  __device__ __forceinline__ uint32_t word(int i) const {
    constexpr int W = sizeof(word_t) / 4;
    return w[i / W][i % W];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (BF16) return __uint_as_float((i & 1) ? (word(i >> 1) & 0xffff0000u) : (word(i >> 1) << 16));
    else return __uint_as_float(word(i));
  }
  __device__ __forceinline__ void set(const float (&v)[V]) {
    constexpr int W = sizeof(word_t) / 4;
    if constexpr (!BF16) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i / W][i % W] = __float_as_uint(v[i]);
    } else if constexpr (V == 1) {
      w[0][0] = f32_to_bf16_rne(v[0]);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) w[i / W][i % W] = f32_to_bf16_rne(v[2 * i]) | (f32_to_bf16_rne(v[2 * i + 1]) << 16);
    }
  }
};

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
    Elems<V, BF16> e0, e1;
    e0.load(src + ES * c0);
    e1.load(src + ES * c1);
    if (turn) {
      float o0[V], o1[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (LAYOUT == CG_ROPE_HALF) {
          const float x0 = e0.get(i), x1 = e1.get(i);
          o0[i] = fmaf(x0, cn[i], -(x1 * sn[i]));
          o1[i] = fmaf(x0, sn[i], x1 * cn[i]);
        } else {  // pairs (2 i, 2 i + 1) of the unit's 2 V channels
          const float x0 = 2 * i < V ? e0.get(2 * i < V ? 2 * i : 0) : e1.get(2 * i < V ? 0 : 2 * i - V);
          const float x1 = 2 * i + 1 < V ? e0.get(2 * i + 1 < V ? 2 * i + 1 : 0) : e1.get(2 * i + 1 < V ? 0 : 2 * i + 1 - V);
          const float y0 = fmaf(x0, cn[i], -(x1 * sn[i])), y1 = fmaf(x0, sn[i], x1 * cn[i]);
          if (2 * i < V) o0[2 * i < V ? 2 * i : 0] = y0;
          else o1[2 * i < V ? 0 : 2 * i - V] = y0;
          if (2 * i + 1 < V) o0[2 * i + 1 < V ? 2 * i + 1 : 0] = y1;
          else o1[2 * i + 1 < V ? 0 : 2 * i + 1 - V] = y1;
        }
      }
      e0.set(o0);
      e1.set(o1);
    }
    e0.store(dst + ES * c0);
    e1.store(dst + ES * c1);
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

hipError_t launch_rope(const cg_rope_plan& plan, const ViewDev& x0, const ViewDev& y0, const ViewDev& x1, const ViewDev& y1,
                       const int* pos, bool inverse, hipStream_t st) {
  RopeArgs a;
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
  if (tokens == 0 || a.skip == 0) return hipSuccess;
  const int64_t blocks = (tokens * a.units + 255) / 256;
  if (tokens * a.units > 0x7fffff00) return hipErrorInvalidValue;
  // rows per thread: as many as leave about four workgroups per CU, at most 8 (8192 tokens x 40 heads: one 41 us, up to
  // four 31.6, eight 30.0, sixteen 30.1; eight workgroups per CU 31.1)
  a.per = int(std::max<int64_t>(1, std::min<int64_t>(8, blocks * rows / (4 * cu_count()))));
  const int gy = (rows + a.per - 1) / a.per;
  if (gy > 65535) return hipErrorInvalidValue;
  const void* fn = x0.bf16 ? rope_by_width<true>(V, plan.layout) : rope_by_width<false>(V, plan.layout);
  void* args[] = {&a};
  return hipLaunchKernel(fn, dim3(unsigned(blocks), gy), dim3(256), args, 0, st);
}

}  // namespace cg
