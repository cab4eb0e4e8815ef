// Chunk attention, bf16 results, rows of 129 to 256 channels.
#include "cg_chunk_kernel.h"

namespace cg {

hipError_t run_chunk_256(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  return by_layout<256, 1, false>(a, G, c, blocks, st);
}

}  // namespace cg
