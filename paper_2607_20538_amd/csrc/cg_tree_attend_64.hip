// Attention of trees, bf16 results, rows of 64 channels.
#include "cg_tree_kernel.h"

namespace cg {

hipError_t run_tree_attend_64(const TreeRun& a, int bits, int qt, int blocks, hipStream_t st) {
  return qt == 1 ? tree_by_bits<64, 1>(a, bits, blocks, st) : tree_by_bits<64, 2>(a, bits, blocks, st);
}

}  // namespace cg
