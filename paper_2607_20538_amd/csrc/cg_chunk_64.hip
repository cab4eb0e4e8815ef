// Chunk attention, bf16 results, rows of at most 64 channels.
#include "cg_chunk_kernel.h"

namespace cg {

hipError_t run_chunk_64(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  return by_layout<64, 1, true>(a, G, c, blocks, st);
}

}  // namespace cg
