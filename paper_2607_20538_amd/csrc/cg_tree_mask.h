// What a node of a tree of drafted tokens sees (one copy per translation unit).
#pragma once

#include "cg_internal.h"

namespace cg {
namespace {

__device__ __forceinline__ uint64_t bits_below(int x) { return x <= 0 ? 0ull : (x >= 64 ? ~0ull : (1ull << x) - 1ull); }

// 64 bits of `nodes` (words) from bit `at` on; what lies outside is zero
__device__ __forceinline__ uint64_t mask_bits(const uint64_t* nodes, int words, int at) {
  const int w = at >> 6, s = at & 63;  // (rounds down)
  const uint64_t lo = w >= 0 && w < words ? nodes[w] : 0, hi = s && w + 1 >= 0 && w + 1 < words ? nodes[w + 1] : 0;
  return s ? (lo >> s) | (hi << (64 - s)) : lo;
}

// Bit c: position t + c is seen.  Of the positions before `base` (what the row held) those after `plow` or below
// `sinks`, of the others, up to `held`, the nodes of the token's mask.
__device__ __forceinline__ uint64_t tree_seen(const uint64_t* nodes, int words, int base, int held, int plow, int sinks, int t) {
  uint64_t seen = bits_below(base - t) & (~bits_below(plow - t + 1) | bits_below(sinks - t));
  if (t + 63 >= base) seen |= mask_bits(nodes, words, t - base) & ~bits_below(base - t) & bits_below(held - t);
  return seen;
}

__device__ __forceinline__ int wave_most(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o));
  return __builtin_amdgcn_readfirstlane(v);
}

}  // namespace
}  // namespace cg
