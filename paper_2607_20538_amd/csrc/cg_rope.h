// Rotations: sine and cosine of the angles, the turn of a thread's channels (one copy per translation unit; the
// angles and the split: cg_rope.hip).
#pragma once

#include "cg_internal.h"
#include "cg_device.h"

namespace cg {

struct RopeArgs {
  cg_rope_plan plan;
  ViewDev x[2], y[2];   // queries and keys (the second may be absent: H = 0)
  const int* pos;       // [B][T]
  int inverse, per;     // rows (layer, head) of a thread
  int units, skip;      // units of 2 V channels a row has; units from `skip` on are left (in-place: nothing to copy)
};
// A rotation's workgroups of 256 threads (gx = 0: nothing to do) and the pairs V that a thread takes
struct RopeSplit {
  RopeArgs a;
  int V;
  unsigned gx, gy;
};
// false: more than a launch holds
bool rope_split(const cg_rope_plan& plan, const ViewDev& x0, const ViewDev& y0, const ViewDev& x1, const ViewDev& y1,
                const int* pos, bool inverse, RopeSplit& s);
hipError_t launch_rope_split(const RopeSplit& s, hipStream_t st);

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

// One row of a thread's channels: the V from c0 and the V from c1, turned
template <int V, bool BF16, int LAYOUT>
__device__ __forceinline__ void turn_row(const char* src, char* dst, int c0, int c1, bool turn, const float (&sn)[V], const float (&cn)[V]) {
  constexpr int ES = BF16 ? 2 : 4;
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
// Workgroup (bx, by) of the split of one view
template <int V, bool BF16, int LAYOUT>
__device__ __forceinline__ void rope_unit(const RopeArgs& a, int bx, int by) {
  constexpr int ES = BF16 ? 2 : 4;
  const ViewDev &X = a.x[0], &Y = a.y[0];
  const int idx = bx * 256 + int(threadIdx.x), u = idx % a.units, tk = idx / a.units;
  if (tk >= X.B * X.T || u >= a.skip) return;
  const int b = tk / X.T, t = tk - b * X.T, p = a.pos[tk], hr = a.plan.d_rot / 2;
  if (p < 0) return;
  const bool turn = u < hr / V;
  float sn[V], cn[V];
  if (turn) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      pair_turn(a.plan, u * V + i, p, sn[i], cn[i]);
      if (a.inverse) sn[i] = -sn[i];
    }
  }
  const int c0 = LAYOUT == CG_ROPE_HALF && turn ? u * V : 2 * u * V;
  const int c1 = LAYOUT == CG_ROPE_HALF && turn ? hr + u * V : c0 + V;
  const int r1 = min(X.L * X.H, (by + 1) * a.per);
#pragma unroll 2
  for (int r = by * a.per; r < r1; ++r) {
    const int lv = r / X.H, h = r - lv * X.H;
    turn_row<V, BF16, LAYOUT>(static_cast<const char*>(X.ptr) + ES * (lv * X.sl + b * X.sb + h * X.sh + t * X.st),
                              static_cast<char*>(Y.ptr) + ES * (lv * Y.sl + b * Y.sb + h * Y.sh + t * Y.st), c0, c1, turn, sn, cn);
  }
}

}  // namespace
}  // namespace cg
