// Chunk attention, binary32 results.
#include "cg_chunk_kernel.h"

namespace cg {

hipError_t run_chunk_f32(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  if (a.q.d <= 64) return by_layout<64, 2, false>(a, G, c, blocks, st);
  if (a.q.d <= 128) return by_layout<128, 2, false>(a, G, c, blocks, st);
  return by_layout<256, 2, false>(a, G, c, blocks, st);
}

}  // namespace cg
