// Attention of trees by the chunk kernel, bf16 results, rows of more than 128 channels.
#include "cg_chunk_kernel.h"

namespace cg {

hipError_t run_tree_256(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  return by_layout<256, 1, false, true>(a, G, c, blocks, st);
}

}  // namespace cg
