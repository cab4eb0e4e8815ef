// Kernel arguments and plan of the chunk attention.
#pragma once

#include "cg_internal.h"

namespace cg {

struct ChunkDev {
  ViewDev q, o;          // [nl][1][Hq][N][d], packed tokens
  CacheDev kc, vc;       // page pools
  PageDev pt;
  int l0, Hq, grp;       // cache layer of view layer 0, query heads, query heads per KV head
  int B, N, max_q;       // batch rows, packed tokens, tokens of a row at most
  int min_q;             // rows with fewer tokens are left (the single-token attention takes them)
  const int* cu;         // device [B + 1] first token of every row
  const int* lens;       // device [B] positions a row holds, its new tokens among them
  float scale;
  int window, sinks;
  int cap;               // positions a row can hold
  int tq, heads, nqc, ntile, nsplit;  // the plan
  float *part, *ml;      // splits: [nl][nsplit][N][Hq][d], [nl][nsplit][N][Hq][2] (maximum, sum)
  int* err;
};

// Rows that decode in runs of 32 channels with one side word each; everything else goes four channels at a time
inline bool chunk_wide(const CodecDev& c, int d) {
  return c.backend == CG_BACKEND_BLOCK_UNIFORM && c.n % 32 == 0 && d % 32 == 0;
}

constexpr int kChunkWaves = 4;  // waves of 32 query rows per workgroup

struct ChunkPlan {
  int tq = 1, heads = 1; // tokens and query heads of a tile
  int nqc = 1;           // chunks of a KV head's query heads
  int ntile = 0;         // tiles at most
  int nsplit = 1;        // parts of a tile's positions
  size_t ws_bytes = 0;
};
// Rows of partial sums that the splits of a plan have at most (layers x splits x tokens x query heads): eight workgroups
// of 128 for every CU.  Splits past that take less than 3% off the last round, at any length of the rows.
inline int64_t chunk_part_rows() { return int64_t(8) * 32 * kChunkWaves * cu_count(); }
constexpr int kChunkSplits = 64;  // parts at most, each of eight steps at least
// singles: rows of one token have another kernel
ChunkPlan chunk_plan(int nl, int N, int B, int max_q, int H, int Hq, int d, int cap, int window, int sinks, bool singles);
// The kernels by rounded row width and result type
hipError_t run_chunk_64(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st);
hipError_t run_chunk_128(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st);
hipError_t run_chunk_256(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st);
hipError_t run_chunk_f32(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st);
hipError_t launch_chunk(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, hipStream_t st);

}  // namespace cg
