// Chunk attention: plan, launch, and the joining of splits (the kernel: cg_chunk_kernel.h).
#include <algorithm>

#include "cg_chunk.h"
#include "cg_chunk_rows.h"
#include "cg_device.h"

namespace cg {

namespace {

// Splits of a tile's steps joined: out = sum_s w_s o_s / sum_s w_s, w_s = l_s 2^(m_s - max m).  One wave per
// (token, query head); a split that saw nothing has l = 0 and its sums are zeros.
__global__ __launch_bounds__(256) void chunk_join(ChunkDev a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = a.q.d;
  const int tile = blockIdx.x % a.ntile, lv = blockIdx.x / a.ntile;
  const QTile qt = find_tile(a, tile);
  if (qt.b < 0) return;
  const int rows = min(a.tq, qt.n - qt.i0) * a.Hq;
  for (int r = blockIdx.y * 4 + w; r < rows; r += 4 * gridDim.y) {
    const int tok = qt.tok0 + qt.i0 + r / a.Hq, head = r % a.Hq;
    auto at = [&](int s) { return ((size_t(lv) * a.nsplit + s) * a.N + tok) * a.Hq + head; };
    float M = -INFINITY;
    for (int s = lane; s < a.nsplit; s += 64) M = fmaxf(M, a.ml[2 * at(s)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    float L = 0.0f;
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int ch = 4 * lane;
    for (int s = 0; s < a.nsplit; ++s) {
      const float ms = a.ml[2 * at(s)], l = a.ml[2 * at(s) + 1];
      const float wt = l == 0.0f ? 0.0f : l * (ms == M ? 1.0f : __builtin_amdgcn_exp2f(ms - M));
      if (wt == 0.0f) continue;
      L += wt;
      if (ch < d) {
        const float4 x = *reinterpret_cast<const float4*>(a.part + at(s) * d + ch);
        y.x = fmaf(wt, x.x, y.x);
        y.y = fmaf(wt, x.y, y.y);
        y.z = fmaf(wt, x.z, y.z);
        y.w = fmaf(wt, x.w, y.w);
      }
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    if (ch >= d) continue;
    const size_t off = size_t(lv) * a.o.sl + size_t(head) * a.o.sh + size_t(tok) * a.o.st + ch;
    y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
    if (a.o.bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.ptr) + off) =
          make_uint2(f32_to_bf16_rne(y.x) | (f32_to_bf16_rne(y.y) << 16), f32_to_bf16_rne(y.z) | (f32_to_bf16_rne(y.w) << 16));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.o.ptr) + off) = y;
  }
}

}  // namespace

ChunkPlan chunk_plan(int nl, int N, int B, int max_q, int H, int Hq, int d, int cap, int window, int sinks) {
  ChunkPlan p;
  const int grp = Hq / H;
  const int64_t mq = std::min(max_q, N);
  const int64_t want_rows = mq * grp;
  p.waves = want_rows <= 32 ? 1 : (want_rows <= 64 ? 2 : 4);
  const int M = 32 * p.waves;
  p.heads = std::min(grp, M);
  p.nqc = (grp + p.heads - 1) / p.heads;
  p.tq = M / p.heads;
  // every row with tokens brings at most one tile that is not full
  const int rows = std::min(N, B);
  p.ntile = int(std::min<int64_t>(int64_t(N) / p.tq + rows, std::min<int64_t>(N, int64_t(rows) * ((mq + p.tq - 1) / p.tq))));
  const int64_t steps = window > 0 ? std::min<int64_t>((int64_t(cap) + kStep - 1) / kStep,
                                                       (int64_t(window) + p.tq + sinks) / kStep + 3)
                                   : (int64_t(cap) + kStep - 1) / kStep;
  const int64_t wgs = int64_t(nl) * H * p.nqc * p.ntile;
  // about 1024 workgroups, each split at least 8 steps (its queries and sums cost about two)
  p.nsplit = int(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((1024 + wgs - 1) / std::max<int64_t>(wgs, 1), steps / 8), 64)));
  p.ws_bytes = p.nsplit > 1 ? size_t(nl) * p.nsplit * N * Hq * (size_t(d) + 2) * sizeof(float) : 0;
  return p;
}

hipError_t launch_chunk(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, hipStream_t st) {
  if (a.N == 0 || a.B == 0 || a.ntile == 0) return hipSuccess;
  const int64_t blocks = int64_t(a.q.L) * a.kc.H * a.nqc * a.ntile * a.nsplit;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  const int d = a.q.d;
  const bool wide = !a.o.bf16;  // binary32 results
  hipError_t e;
  if (wide) e = run_chunk_f32(a, G, c, int(blocks), st);
  else if (d <= 64) e = run_chunk_64(a, G, c, int(blocks), st);
  else if (d <= 128) e = run_chunk_128(a, G, c, int(blocks), st);
  else e = run_chunk_256(a, G, c, int(blocks), st);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int per = std::min(16, (a.tq * a.Hq + 3) / 4);
  hipLaunchKernelGGL(chunk_join, dim3(a.ntile * a.q.L, per), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace cg
