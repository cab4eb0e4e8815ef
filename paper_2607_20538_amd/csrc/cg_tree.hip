// Trees of drafted tokens: positions and masks from the nodes' parents, the path that a model agrees with, and
// the entries of that path moved together in the page pools.
//
// Row b's nodes are packed tokens [cu[b], cu[b + 1]); parent[i] is the parent of a node within its row (-1: a root), below the
// node itself, so every path ascends.  All three are bound by latency: a few dependent loads per row.
#include <algorithm>

#include "cg_internal.h"

namespace cg {

namespace {

constexpr int kTreeThreads = 256;

// The row's nodes, or -1: cu runs backwards, past the packed tokens, or over `most` nodes
__device__ __forceinline__ int row_nodes(const int* cu, int b, int N, int most, int& first) {
  first = cu[b];
  const int n = cu[b + 1] - first;
  return first < 0 || n < 0 || first > N - n || n > most ? -1 : n;
}

// First token behind all rows: cu[B], or where rows run backwards (other workgroups write the tokens of those before
// them) the largest of cu.  By each wave for itself
__device__ __forceinline__ int rows_end(const int* cu, int B, int N) {
  int end = cu[B];
  if (end < N) {
    for (int b = threadIdx.x & 63; b < B; b += 64) end = max(end, cu[b]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) end = max(end, __shfl_xor(end, o));
  }
  return min(max(end, 0), N);
}

// ------------------------------------------------------------------------------------------
// positions and masks
// ------------------------------------------------------------------------------------------
// One workgroup per row.  A thread walks a node's ancestors inside the node's own 64-bit word (`up` in LDS), which
// gives that word and the first ancestor below it; then from word to word, whole words at a time.  So a node
// takes at most 64 + n / 64 dependent LDS reads, a shallow one as many as its depth.  32 trees of 16 nodes 2.8 us, 256 of up
// to 250 (1.5 MB of masks) 3.5: little more than a launch.
//
// A window hides ancestors as it hides held positions: of a node at depth k, position base + k, those at depths from
// sinks - base up to k - window.  Ancestors lie in order of their depth in a mask (a parent is an earlier node), so they
// are a run of its set bits; the depth is counted before the words are written (WINDOW: the 256 rows of up to 250 nodes
// 3.6 us, as chains 5.4 to 7.2, without a window 4.9).
struct TreeMapArgs {
  const int *parent, *cu, *lens;
  int B, N, words, window, sinks;
  int* pos;
  uint64_t* mask;
  int* err;
};

// m without its set bits of rank lo .. hi - 1, counted from the lowest
__device__ __forceinline__ uint64_t without_ranks(uint64_t m, int lo, int hi) {
  uint64_t x = m;
  for (int i = 0; i < lo; ++i) x &= x - 1;
  uint64_t y = x;
  for (int i = lo; i < hi; ++i) y &= y - 1;
  return (m ^ x) | y;
}

template <bool WINDOW>
__global__ __launch_bounds__(kTreeThreads) void tree_map(TreeMapArgs a) {
  __shared__ int up[CG_TREE_MOST];         // parent
  __shared__ uint64_t own[CG_TREE_MOST];   // ancestors (and itself) in the node's word
  __shared__ int out[CG_TREE_MOST];        // its first ancestor below that word, -1: none
  const int b = blockIdx.x, tid = threadIdx.x;
  if (b == a.B) {  // behind the last row
    const int end = rows_end(a.cu, a.B, a.N);
    for (int64_t x = int64_t(end) * a.words + tid; x < int64_t(a.N) * a.words; x += kTreeThreads) a.mask[x] = 0;
    for (int i = end + tid; i < a.N; i += kTreeThreads) a.pos[i] = -1;
    return;
  }
  int first;
  const int n = row_nodes(a.cu, b, a.N, min(64 * a.words, CG_TREE_MOST), first);
  if (n < 0) {
    if (tid == 0 && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
    return;
  }
  const int len = a.lens[b], base = len < n ? -1 : len - n;  // (any int may stand there)
  bool bad = base < 0;
  for (int i = tid; i < n; i += kTreeThreads) {
    int p = a.parent[first + i];
    if (p < -1 || p >= i) {
      bad = true;
      p = -1;
    }
    up[i] = p;
  }
  if (bad && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
  __syncthreads();
  for (int i = tid; i < n; i += kTreeThreads) {
    uint64_t m = 0;
    int x = i;
    do {
      m |= uint64_t(1) << (x & 63);
      x = up[x];
    } while (x >= (i & ~63));
    own[i] = m;
    out[i] = x;
  }
  __syncthreads();
  const int shown = WINDOW ? min(max(a.sinks - max(base, 0), 0), n) : 0;  // depths that are sinks
  for (int i = tid; i < n; i += kTreeThreads) {
    uint64_t* dst = a.mask + size_t(first + i) * a.words;
    int depth = -1;
    if constexpr (WINDOW) {
      for (int x = i; x >= 0; x = out[x]) depth += __popcll(own[x]);
    }
    const int hidden = depth - a.window + 1;  // ancestors at depths below, where there is a window
    int left = depth + 1, x = i, w = a.words - 1;
    while (x >= 0) {
      for (; w > x >> 6; --w) dst[w] = 0;
      uint64_t m = own[x];
      if constexpr (WINDOW) {
        const int k = __popcll(m);
        left -= k;  // depth of the word's first
        m = without_ranks(m, min(max(shown - left, 0), k), min(max(hidden - left, 0), k));
      } else {
        depth += __popcll(m);
      }
      dst[w--] = m;
      x = out[x];
    }
    for (; w >= 0; --w) dst[w] = 0;
    a.pos[first + i] = base < 0 ? -1 : base + depth;
  }
}

// ------------------------------------------------------------------------------------------
// the path that the model agrees with
// ------------------------------------------------------------------------------------------
// One wave per row: from a kept node the lowest child whose draft is the model's choice there, found by a ballot over 64 nodes at
// a time from the node on (children follow their parent, so a whole walk looks at every node about once).  32 trees of 16
// nodes 3.2 us, 256 of up to 250 nodes 4.5.
struct TreeAcceptArgs {
  const int *parent, *cu, *draft, *target, *head;
  int B, N;
  int *path, *kept, *next;
  int* err;
};

__global__ __launch_bounds__(64) void tree_accept(TreeAcceptArgs a) {
  __shared__ int up[CG_TREE_MOST], said[CG_TREE_MOST];
  const int b = blockIdx.x, lane = threadIdx.x;
  if (b == a.B) {
    for (int i = rows_end(a.cu, a.B, a.N) + lane; i < a.N; i += 64) a.path[i] = -1;
    return;
  }
  int first;
  const int n = row_nodes(a.cu, b, a.N, CG_TREE_MOST, first);
  if (n < 0) {
    if (lane == 0) {
      if (a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
      a.kept[b] = 0;
      a.next[b] = -1;
    }
    return;
  }
  bool bad = false;
  for (int i = lane; i < n; i += 64) {
    const int p = a.parent[first + i];
    bad |= p < -1 || p >= i;
    up[i] = p;
    said[i] = a.draft[first + i];
  }
  if (bad && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
  __syncthreads();
  int at = -1, kept = 0;
  bool any = !a.head;  // the first root is taken, whatever it drafts
  int want = a.head ? a.head[b] : -1;
  for (int i0 = 0; i0 < n;) {
    const int i = i0 + lane;
    // (a parent that is none of the earlier nodes makes its node unreachable)
    const bool hit = i < n && i > at && up[i] == at && (any || said[i] == want);
    const uint64_t found = __builtin_amdgcn_ballot_w64(hit);
    if (!found) {
      i0 += 64;
      continue;
    }
    at = i0 + __builtin_ctzll(found);
    want = a.target[first + at];
    any = false;
    if (lane == 0) a.path[first + kept] = at;
    ++kept;
  }
  for (int i = kept + lane; i < n; i += 64) a.path[first + i] = -1;
  if (lane == 0) {
    a.kept[b] = kept;
    a.next[b] = want;
  }
}

// ------------------------------------------------------------------------------------------
// the path's entries moved together
// ------------------------------------------------------------------------------------------
// Entry base + path[j] of a row goes to base + j in every layer and head of both pools.  path ascends, so a place is written
// only after it was read where no batch is written before all of it is read: a later batch reads behind all places of
// the earlier ones.  A workgroup takes one row and some (pool, layer, head) slices; its threads take the 16-byte (8, 4)
// pieces of the entries that move, kPieces reads in flight each.  Latency: the row's path, its pages, one read and one write.  64
// rows of 60 nodes in 8 layers of 16 heads at 4 bits: 8.6 us; 32 rows of 16 in 4 layers of error-free pools: 7.2.
constexpr int kPieces = 4;

struct TreeKeepArgs {
  const int *path, *kept, *cu, *lens;
  PageDev pt;
  CacheDev k[2];
  int l0, nl, B, N;
  int row_bytes, side_words;  // of an entry
  int unit;                   // bytes of a piece of its codes
  int per, groups;            // slices of a workgroup, workgroups of a row
  int* held;
  int* err;
};

template <typename T>
__device__ __forceinline__ void tree_move(const TreeKeepArgs& a, const int2* move, int count, int s0, int s1) {
  const int cu = a.row_bytes / int(sizeof(T)), U = cu + a.side_words;  // pieces of an entry
  const int H = a.k[0].H, P = a.k[0].T_cap, tid = threadIdx.x;
  constexpr int CAP = kTreeThreads * kPieces;
  const int most = max(1, CAP / U);              // entries of a batch
  const int ne = min(count, most);               // ... of one slice
  const int ns = max(1, min(s1 - s0, most / ne)); // slices of a batch
  for (int s = s0; s < s1; s += ns) {
    for (int e0 = 0; e0 < count; e0 += ne) {
      const int ents = min(ne, count - e0), items = min(ns, s1 - s) * ents * U;
      T v[kPieces];
      char* dst[kPieces];
      bool code[kPieces];
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        const int x = tid + q * kTreeThreads;
        v[q] = T{};
        dst[q] = nullptr;
        code[q] = false;
        if (x < items) {
          const int u = x % U, y = x / U, e = e0 + y % ents, sl = s + y / ents;
          const int h = sl % H, lp = sl / H, pool = lp & 1, l = a.l0 + (lp >> 1);
          const CacheDev& k = a.k[pool];
          auto row = [&](int slot) {
            const int pg = slot / P;
            return ((size_t(l) * k.B + pg) * H + h) * P + (slot - pg * P);
          };
          const int2 m = move[e];
          if (m.x >= 0 && m.y >= 0) {
            code[q] = u < cu;
            if (code[q]) {
              v[q] = *reinterpret_cast<const T*>(k.codes + row(m.x) * a.row_bytes + size_t(u) * sizeof(T));
              dst[q] = reinterpret_cast<char*>(k.codes + row(m.y) * a.row_bytes + size_t(u) * sizeof(T));
            } else {
              *reinterpret_cast<uint32_t*>(&v[q]) = k.side[row(m.x) * a.side_words + (u - cu)];
              dst[q] = reinterpret_cast<char*>(k.side + row(m.y) * a.side_words + (u - cu));
            }
          }
        }
      }
      // everything read has arrived before anything is written
#pragma unroll
      for (int q = 0; q < kPieces; ++q) asm volatile("" ::"v"(*reinterpret_cast<const uint32_t*>(&v[q])));
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        if (!dst[q]) continue;
        if (code[q]) *reinterpret_cast<T*>(dst[q]) = v[q];
        else *reinterpret_cast<uint32_t*>(dst[q]) = *reinterpret_cast<const uint32_t*>(&v[q]);
      }
    }
  }
}

__global__ __launch_bounds__(kTreeThreads) void tree_keep(TreeKeepArgs a) {
  __shared__ int2 move[CG_TREE_MOST];  // slots that move, from and to (-1: outside the pool)
  const int b = blockIdx.x / a.groups, grp = blockIdx.x - b * a.groups, tid = threadIdx.x;
  int first;
  const int n = row_nodes(a.cu, b, a.N, CG_TREE_MOST, first);
  const int len = a.lens[b], kept = a.kept[b], base = n < 0 || len < n ? -1 : len - n, P = a.pt.page_size;
  bool ok = base >= 0 && kept >= 0 && kept <= n && len <= int64_t(a.pt.max_pages) * P;
  int stay = 0;  // nodes at their places: the first ones
  bool fine = true, out = false;
  for (int j = tid; ok && j < kept; j += kTreeThreads) {
    const int at = a.path[first + j], before = j ? a.path[first + j - 1] : -1;
    if (at <= before || at >= n) fine = false;
    stay += at == j;
  }
  ok = __syncthreads_and(fine) && ok;
  if (!ok) {  // nothing of the row is kept of what was added, where that is known
    if (tid == 0 && grp == 0) {
      if (a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
      a.held[b] = base >= 0 ? base : len;
    }
    return;
  }
  if (tid == 0 && grp == 0) a.held[b] = base + kept;
  // the sum over the workgroup
  __shared__ int total;
  if (tid == 0) total = 0;
  __syncthreads();
  if (stay) atomicAdd(&total, stay);
  __syncthreads();
  stay = total;
  const int count = kept - stay;
  auto slot = [&](int p) {
    const int pg = a.pt.pages[size_t(b) * a.pt.max_pages + p / P];
    if (pg < 0 || pg >= a.k[0].B) {
      out = true;
      return -1;
    }
    return pg * P + p % P;
  };
  for (int j = tid; j < count; j += kTreeThreads) move[j] = make_int2(slot(base + a.path[first + stay + j]), slot(base + stay + j));
  if (out && grp == 0 && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
  __syncthreads();
  if (count == 0) return;
  const int s0 = grp * a.per, s1 = min(2 * a.nl * a.k[0].H, s0 + a.per);
  if (a.unit == 16) tree_move<uint4>(a, move, count, s0, s1);
  else if (a.unit == 8) tree_move<uint2>(a, move, count, s0, s1);
  else tree_move<uint32_t>(a, move, count, s0, s1);
}

}  // namespace

hipError_t launch_tree_map(const int* parent, const int* cu, const int* lens, int B, int N, int words, int window, int sinks,
                           int* pos, uint64_t* mask, int* err, hipStream_t st) {
  TreeMapArgs a{parent, cu, lens, B, N, words, window, sinks, pos, mask, err};
  if (window > 0) hipLaunchKernelGGL(tree_map<true>, dim3(B + 1), dim3(kTreeThreads), 0, st, a);
  else hipLaunchKernelGGL(tree_map<false>, dim3(B + 1), dim3(kTreeThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_tree_accept(const int* parent, const int* cu, const int* draft, const int* target, const int* head, int B, int N,
                              int* path, int* kept, int* next, int* err, hipStream_t st) {
  TreeAcceptArgs a{parent, cu, draft, target, head, B, N, path, kept, next, err};
  hipLaunchKernelGGL(tree_accept, dim3(B + 1), dim3(64), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_tree_keep(const int* path, const int* kept, const int* cu, const int* lens, int B, int N, const PageDev& pt,
                            const CodecDev& c, const CacheDev& kc, const CacheDev& vc, int l0, int nl, int* held, int* err,
                            hipStream_t st) {
  TreeKeepArgs a;
  a.path = path;
  a.kept = kept;
  a.cu = cu;
  a.lens = lens;
  a.pt = pt;
  a.k[0] = kc;
  a.k[1] = vc;
  a.l0 = l0;
  a.nl = nl;
  a.B = B;
  a.N = N;
  const bool pass = c.backend == CG_BACKEND_PASSTHROUGH;
  a.row_bytes = pass ? 4 * kc.d : kc.d * c.bits / 8;
  a.side_words = pass ? 0 : kc.d / c.n;
  a.unit = a.row_bytes % 16 == 0 ? 16 : (a.row_bytes % 8 == 0 ? 8 : 4);
  a.held = held;
  a.err = err;
  // slices of a workgroup: as many as leave about eight workgroups per CU
  const int64_t slices = int64_t(2) * nl * kc.H;
  a.per = int(std::max<int64_t>(1, std::min<int64_t>(slices, slices * B / (8 * int64_t(cu_count())))));
  a.groups = int((slices + a.per - 1) / a.per);
  if (int64_t(a.groups) * B > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(tree_keep, dim3(unsigned(a.groups * B)), dim3(kTreeThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace cg
