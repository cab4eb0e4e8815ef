// Chunk attention, bf16 results, rows of 65 to 128 channels.
#include "cg_chunk_kernel.h"

namespace cg {

hipError_t run_chunk_128(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  return by_layout<128, 1, true>(a, G, c, blocks, st);
}

}  // namespace cg
