// Kernel arguments, plan and workspace of the attention of trees (kernels: cg_tree_kernel.h, cg_tree_join.hip).
#pragma once

#include "cg_chunk.h"

namespace cg {

constexpr int kTreeBlock = 128;  // positions that the four waves of a workgroup take at a time, 32 each

// A tile: up to 32 QT query rows (tokens x query heads of a KV head) of one batch row.  Its place on the line of all tiles'
// blocks of positions: [start, start + len), the first kTileCost of them no blocks but what the tile costs beside them.
constexpr int kTileCost = 2;
struct TreeTile {
  int64_t start;
  int len, b, tok0, ntok;  // blocks, batch row, first packed token, tokens
  int base, held;          // positions before the row's new tokens, and with them (a row that cannot be taken: 0, 0)
  int wg0, wg1;            // first and last workgroup on it
};
// Order of a run of 32 channels in operands: dword j of granule g holds the channels of part 0 and 1: 4, 3 and 2 bits as
// the bytes of a masked word hold them, other widths as code_pair takes them.
__host__ __device__ constexpr int tree_channel(int bits, int g, int j, int part) {
  return bits == 4   ? 8 * g + 4 * (j & 1) + (j >> 1) + 2 * part
         : bits == 3 ? 2 * g + (j >> 1) + 16 * (j & 1) + 8 * part
         : bits == 2 ? 8 * g + j + 4 * part
                     : 16 * (g >> 1) + 4 * (g & 1) + j + 8 * part;
}
struct TreeLine {
  int64_t total, per;  // blocks of the line, and of a workgroup
};

struct TreeDev {
  ChunkDev c;          // tq, heads, nqc: of the tiles; ntile: room for tiles
  int bits, qt, nwg;   // code width, groups of 32 query rows of a tile, workgroups per (layer, KV head, chunk of heads)
  // workspace
  TreeLine* line;
  TreeTile* tiles;     // [ntile], len 0 behind the last
  int* first;          // [nwg] the tile that a workgroup begins in
  uint4* qf;           // [nl][H][nqc][ntile][qt][d / 16][64] operands of the gauged queries
  float* qs;           // [nl][H][nqc][ntile][32 qt] what their scores are scaled by
  float* part;         // [nl][H][nqc][nwg + ntile][qt][d / 32][4][64][4] sums of (workgroup w, tile t) at w + t
  float2* ml;          // [nl][H][nqc][nwg + ntile][32 qt] their maxima and sums of weights
};

// What the kernel over the positions takes of it
struct TreeRun {
  const uint8_t *kcodes, *vcodes;
  const uint32_t *kside, *vside;
  const int* pages;
  const uint64_t* mask;
  const int* pos;
  int* err;
  const TreeLine* line;
  const TreeTile* tiles;
  const int* first;
  const uint4* qf;
  const float* qs;
  float* part;
  float2* ml;
  int l0, H, nqc, heads, grp, n, page_size, max_pages, pages_all, words, window, sinks, ntile, nwg;
};

struct TreePlan {
  int qt = 1, tq = 1, heads = 1, nqc = 1, ntile = 0, nwg = 1;
  size_t off_tiles = 0, off_first = 0, off_qf = 0, off_qs = 0, off_part = 0, off_ml = 0, bytes = 0;
};
// Whether the kernels take these pools, views and heads
bool tree_attend_supported(const CodecDev& c, int d, int grp, bool bf16_out);
TreePlan tree_plan(int nl, int N, int B, int max_q, int H, int Hq, int d);
// Bytes that every plan of at most these sizes stays within
double tree_plan_limit(int nl, int N, int B, int H, int Hq, int d);
hipError_t run_tree_attend_64(const TreeRun& a, int bits, int qt, int blocks, hipStream_t st);
hipError_t run_tree_attend_128(const TreeRun& a, int bits, int qt, int blocks, hipStream_t st);
hipError_t launch_tree_attend(const ChunkDev& a, const TreePlan& p, void* ws, const GaugeDev& G, const CodecDev& c, hipStream_t st);

}  // namespace cg
