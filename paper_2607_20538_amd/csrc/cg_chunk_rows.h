// Which tokens a workgroup of the chunk attention takes (one copy per translation unit).
#pragma once

#include "cg_chunk.h"

namespace cg {
namespace {

constexpr int kStep = 64;  // positions per step

// The tile-th query tile of the batch: its row, the row's tokens and which of them the tile takes.  Every row
// brings ceil(n_b / tq) tiles, in order; within a row the last tile (which sees the most) comes first.
struct QTile {
  int b = -1, tok0 = 0, n = 0, i0 = 0;  // row (-1: past the last tile), first packed token, tokens, first of the tile
};
__device__ __forceinline__ int row_tokens(const ChunkDev& a, int b, int& c0) {
  c0 = a.cu[b];
  const int n = a.cu[b + 1] - c0;
  return c0 < 0 || n < 0 || c0 > a.N - n || n > a.max_q ? -1 : n;
}
__device__ __forceinline__ QTile find_tile(const ChunkDev& a, int tile) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  QTile r;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int c0 = 0, n = 0;
    if (b0 + lane < a.B) n = row_tokens(a, b0 + lane, c0);
    if (n < a.min_q) n = 0;
    const int nt = (n + a.tq - 1) / a.tq;
    int sum = nt;  // inclusive prefix sum over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o);
      if (lane >= o) sum += v;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(tile < before + sum);
    if (hit) {
      const int src = __builtin_ctzll(hit);
      const int first = before + __shfl(sum, src) - __shfl(nt, src);
      r.b = b0 + src;
      r.tok0 = __shfl(c0, src);
      r.n = __shfl(n, src);
      r.i0 = (__shfl(nt, src) - 1 - (tile - first)) * a.tq;
      break;
    }
    before += __shfl(sum, 63);
  }
  r.b = __builtin_amdgcn_readfirstlane(r.b);
  r.tok0 = __builtin_amdgcn_readfirstlane(r.tok0);
  r.n = __builtin_amdgcn_readfirstlane(r.n);
  r.i0 = __builtin_amdgcn_readfirstlane(r.i0);
  return r;
}

}  // namespace
}  // namespace cg
