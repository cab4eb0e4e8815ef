// Chunk attention: plan, launch, and the joining of splits (the kernel: cg_chunk_kernel.h).
#include <algorithm>
#include <cmath>

#include "cg_chunk.h"
#include "cg_chunk_rows.h"
#include "cg_device.h"

namespace cg {

namespace {

// Splits of a tile's steps joined: out = sum_s w_s o_s / sum_s w_s, w_s = l_s 2^(m_s - max m).  One wave per
// (token, query head), its lanes first the splits' weights (at most 64), then four channels each; a split that saw
// nothing has l = 0.  64 tokens x 32 heads x 32 splits: 198 us with 16 rows per wave and a chain of reads, 10 so.
__global__ __launch_bounds__(256) void chunk_join(ChunkDev a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = a.q.d;
  const int tile = blockIdx.x % a.ntile, lv = blockIdx.x / a.ntile;
  const QTile qt = find_tile(a, tile);
  if (qt.b < 0) return;
  const int rows = min(a.tq, qt.n - qt.i0) * a.Hq;
  for (int r = blockIdx.y * 4 + w; r < rows; r += 4 * gridDim.y) {
    const int tok = qt.tok0 + qt.i0 + r / a.Hq, head = r % a.Hq;
    auto at = [&](int s) { return ((size_t(lv) * a.nsplit + s) * a.N + tok) * a.Hq + head; };
    float m = -INFINITY, l = 0.0f;
    if (lane < a.nsplit) {
      const float2 v = *reinterpret_cast<const float2*>(a.ml + 2 * at(lane));
      m = v.x;
      l = v.y;
    }
    float M = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float wt = l == 0.0f ? 0.0f : l * (m == M ? 1.0f : __builtin_amdgcn_exp2f(m - M));
    float L = wt;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o);
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const int ch = 4 * lane;
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float* src = a.part + at(0) * d + (ch < d ? ch : 0);
    const size_t next = size_t(a.N) * a.Hq * d;
#pragma unroll 4
    for (int s = 0; s < a.nsplit; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(src + s * next);
      const float ws = __shfl(wt, s);
      if (ws != 0.0f) {  // (0 times an infinity is not 0)
        y.x = fmaf(ws, x.x, y.x);
        y.y = fmaf(ws, x.y, y.y);
        y.z = fmaf(ws, x.z, y.z);
        y.w = fmaf(ws, x.w, y.w);
      }
    }
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

ChunkPlan chunk_plan(int nl, int N, int B, int max_q, int H, int Hq, int d, int cap, int window, int sinks, bool singles) {
  ChunkPlan p;
  const int grp = Hq / H;
  const int64_t mq = std::min(max_q, N);
  constexpr int M = 32 * kChunkWaves;
  p.heads = std::min(grp, M);
  p.nqc = (grp + p.heads - 1) / p.heads;
  p.tq = M / p.heads;
  // every row with tokens brings at most one tile that is not full
  const int rows = std::min(N, B);
  p.ntile = int(std::min<int64_t>(int64_t(N) / p.tq + rows, std::min<int64_t>(N, int64_t(rows) * ((mq + p.tq - 1) / p.tq))));
  const int64_t steps = window > 0 ? std::min<int64_t>((int64_t(cap) + kStep - 1) / kStep,
                                                       (int64_t(window) + p.tq + sinks) / kStep + 3)
                                   : (int64_t(cap) + kStep - 1) / kStep;
  // Splits: the least estimated time in us, from what steps were measured to take (d = 128): 1.7 alone on a CU, 1.33
  // each beside others, queries and sums as much as 6, the sums of splits written and read at 4 TB/s and joined in 5.
  // (bf16 results.  Against the best of 1 to 64 splits, six batches of 16 to 1500 tokens over 2000 to 20000 positions: within
  // 9% for d = 64, 128, 256 and both result types; blocks of 16 channels and error-free pools 35% and 28% at worst.)
  // Of rows with few tokens each is a tile; where single tokens have another kernel, little is known of the others.
  const double tiles = mq == 1 ? rows
                               : std::min<double>(p.ntile, double(N) / p.tq + (singles ? 1 + std::min(rows / 2.0, N / (4.0 * p.tq))
                                                                                      : 0.5 * rows + 0.5));
  const double wgs = tiles * nl * H * p.nqc;
  double best = 0;
  for (int ns = 1; ns <= kChunkSplits && (ns == 1 || (ns * 8 <= steps && int64_t(nl) * N * Hq * ns <= chunk_part_rows())); ++ns) {
    const double w = wgs * ns / cu_count(), k = w <= 3 ? std::ceil(w) : w + 0.2;
    const double t = (k <= 1 ? 1.7 : 1.33 * k) * (double(steps) / ns + 6) + (ns > 1 ? 5 + double(nl) * N * Hq * d * 8 * ns / 4e6 : 0);
    if (ns == 1 || t < best) {
      best = t;
      p.nsplit = ns;
    }
  }
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
  const bool tree = a.mask != nullptr;
  if (wide) e = (tree ? run_tree_f32 : run_chunk_f32)(a, G, c, int(blocks), st);
  else if (d <= 64) e = (tree ? run_tree_64 : run_chunk_64)(a, G, c, int(blocks), st);
  else if (d <= 128) e = (tree ? run_tree_128 : run_chunk_128)(a, G, c, int(blocks), st);
  else e = (tree ? run_tree_256 : run_chunk_256)(a, G, c, int(blocks), st);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int per = std::min(65535, (a.tq * a.Hq + 3) / 4);
  hipLaunchKernelGGL(chunk_join, dim3(a.ntile * a.q.L, per), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace cg
