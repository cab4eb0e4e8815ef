// Block tables and slots of a serving step on the GPU, from the requests' lengths: which pages a row takes
// from the pool, where each new token goes, its position, and the rows' first tokens and new lengths.
//
// With P positions per page a row that holds `held` positions and adds `add` takes the pages
// [ceil(held / P), ceil((held + add) / P)) of its table from the top of the pool's stack of free pages, rows in
// order.  Two prefix sums over the rows (tokens, new pages) say where each row's start; every new page and
// every token then finds its row by bisection, so one long prompt costs what many short ones do.
//
// Bound by latency: a few dependent steps of one workgroup.  The tokens are mapped by the same launch while
// they are few; above kOneLaunch a second launch spreads them over the chip (map_tokens).  With the copy of a count
// beside it: 64 rows of one token 6.5 us, 16 rows of 1024 tokens 9.4; one launch against two 8.5 : 9.4 us at 2048 tokens,
// 10.1 : 9.4 at 4096, 13.5 : 9.4 at 8192, 70 : 10 at 65536.
#include <algorithm>

#include "cg_internal.h"

namespace cg {

namespace {

constexpr int kMapThreads = 1024;
constexpr int kOneLaunch = 2048;  // tokens the first launch maps itself

struct MapArgs {
  const int *held, *add;
  int B, N, max_pages, P, n_pages;
  int *free_pages, *count;
  int *pages, *cu, *lens, *pos, *slots;
  int* err;
};

__device__ __forceinline__ int pages_of(int64_t n, int P) { return int((n + P - 1) / P); }

// inclusive prefix sums of (a, b) over the workgroup; the totals in ta, tb
__device__ __forceinline__ void scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb, int64_t (*sums)[2]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t va = __shfl_up(a, o), vb = __shfl_up(b, o);
    if (lane >= o) {
      a += va;
      b += vb;
    }
  }
  __syncthreads();  // the sums of the call before are read
  if (lane == 63) {
    sums[w][0] = a;
    sums[w][1] = b;
  }
  __syncthreads();
  ta = 0;
  tb = 0;
  for (int i = 0; i < nw; ++i) {
    const int64_t x = sums[i][0], y = sums[i][1];
    if (i < w) {
      a += x;
      b += y;
    }
    ta += x;
    tb += y;
  }
}

// The row of item k of a round: first[row] <= k < first[row + 1]
__device__ __forceinline__ int row_of(const int64_t* first, int64_t k) {
  int lo = 0, hi = kMapThreads;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Token i: its row by bisection of cu (cu[0] = 0 <= i < cu[B]), position and slot
__device__ __forceinline__ void map_token(const MapArgs& a, const int* cu, int i) {
  const int total = cu[a.B];
  int p = -1, slot = -1;
  if (i < total) {
    int lo = 0, hi = a.B;  // cu[lo] <= i < cu[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= i) lo = mid;
      else hi = mid;
    }
    const int len = a.lens[lo], held = len - (cu[lo + 1] - cu[lo]);
    p = held + (i - cu[lo]);
    // (a row with a negative held has no page of its own, and a length that stuck at the largest does not say where the row's
    // tokens go: whatever the table holds belongs to others)
    const int lp = held >= 0 && len < 0x7fffffff ? p / a.P : -1;
    const int pg = lp >= 0 && lp < a.max_pages ? a.pages[size_t(lo) * a.max_pages + lp] : -1;
    if (pg >= 0 && pg < a.n_pages) slot = pg * a.P + (p - lp * a.P);
    else if (a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
  }
  a.pos[i] = p;
  a.slots[i] = slot;
}

__global__ __launch_bounds__(kMapThreads) void map_rows(MapArgs a) {
  __shared__ int64_t sums[kMapThreads / 64][2];
  __shared__ int64_t first[kMapThreads + 1];  // new pages taken before each row of the round
  __shared__ int shad[kMapThreads];           // pages each row of the round had (held may be lens itself)
  __shared__ int scu[kMapThreads + 1];        // cu, when one round holds all rows
  const int tid = threadIdx.x;
  const int have = min(max(*a.count, 0), a.n_pages);
  int64_t tok = 0, taken = 0;  // tokens and new pages of the rounds before
  int flags = 0;
  if (tid == 0) {
    first[0] = 0;
    scu[0] = 0;
    a.cu[0] = 0;
  }
  for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int b = b0 + tid;
    int64_t add = 0, len = 0, fresh = 0;
    int had = 0;
    if (b < a.B) {
      const int held = a.held[b], n = a.add[b];
      if (held < 0 || n < 0) flags |= CG_FLAG_POS_RANGE;
      add = max(n, 0);
      len = held + add;
      if (len > int64_t(a.max_pages) * a.P) flags |= CG_FLAG_POS_RANGE;
      if (held >= 0) {
        had = min(pages_of(held, a.P), a.max_pages);
        fresh = min(pages_of(len, a.P), a.max_pages) - had;
      }
    }
    int64_t tokens, pages;
    scan2(add, fresh, tokens, pages, sums);
    if (b < a.B) {
      // counts past 2^31 - 1 cannot be held: they stick there, flagged
      const int64_t end = tok + add, top = 0x7fffffff;
      if (end > top || len > top) flags |= CG_FLAG_POS_RANGE;
      a.cu[b + 1] = int(min(end, top));
      a.lens[b] = int(min(len, top));
      scu[tid + 1] = int(min(end, top));
    }
    first[tid + 1] = fresh;
    shad[tid] = had;
    __syncthreads();
    // new page k of the round, from the top of the stack
    for (int64_t k = tid; k < pages; k += kMapThreads) {
      const int r = row_of(first, k), i = shad[r] + int(k - first[r]);
      const int64_t s = have - 1 - taken - k;
      const int pg = s >= 0 ? a.free_pages[s] : -1;
      const bool ok = pg >= 0 && pg < a.n_pages;
      if (!ok) flags |= CG_FLAG_POOL_EMPTY;
      a.pages[size_t(b0 + r) * a.max_pages + i] = ok ? pg : -1;
    }
    tok += tokens;
    taken += pages;
    __syncthreads();
  }
  if (tok > a.N) flags |= CG_FLAG_POS_RANGE;  // tokens past the arrays are not mapped
  if (tid == 0) *a.count = int(max(int64_t(0), have - taken));
  if (flags && a.err) atomicOr(a.err, flags);
  if (a.N > kOneLaunch) return;
  __syncthreads();
  for (int i = tid; i < a.N; i += kMapThreads) map_token(a, a.B <= kMapThreads ? scu : a.cu, i);
}

__global__ __launch_bounds__(256) void map_tokens(MapArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < a.N) map_token(a, a.cu, i);
}

// Rows that are done give their pages back: pushed on the stack row by row, their table entries -1, length 0.
// TRIM: `done` holds the positions that each row keeps, and the pages past them are given back.
template <bool TRIM>
__global__ __launch_bounds__(kMapThreads) void release_rows(MapArgs a, const int* done) {
  __shared__ int64_t sums[kMapThreads / 64][2];
  __shared__ int64_t first[kMapThreads + 1];  // table entries of the round's rows before each row
  __shared__ int stay[TRIM ? kMapThreads : 1];  // entries that each row of the round keeps
  const int tid = threadIdx.x;
  int64_t base = min(max(*a.count, 0), a.n_pages);
  int flags = 0;
  if (tid == 0) first[0] = 0;
  for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int b = b0 + tid;
    int64_t n = 0, ok = 0, entries, pushed;
    if constexpr (TRIM) {
      if (b < a.B) {
        const int len = a.lens[b], keep = done[b];
        // (a row that cannot be trimmed stays as it is)
        if (keep < 0 || keep > len || len > int64_t(a.max_pages) * a.P) {
          flags |= CG_FLAG_POS_RANGE;
        } else {
          stay[tid] = pages_of(keep, a.P);
          n = pages_of(len, a.P) - stay[tid];
          a.lens[b] = keep;
        }
      }
    } else if (b < a.B && done[b]) {
      const int len = a.lens[b];
      if (len < 0 || len > int64_t(a.max_pages) * a.P) flags |= CG_FLAG_POS_RANGE;
      n = min(pages_of(max(len, 0), a.P), a.max_pages);
      a.lens[b] = 0;
    }
    scan2(n, ok, entries, pushed, sums);
    first[tid + 1] = n;
    __syncthreads();
    for (int64_t k0 = 0; k0 < entries; k0 += kMapThreads) {
      const int64_t k = k0 + tid;
      int pg = -1;
      if (k < entries) {
        const int r = row_of(first, k);
        int* e = a.pages + size_t(b0 + r) * a.max_pages + int(k - first[r]) + (TRIM ? stay[r] : 0);
        pg = *e;
        *e = -1;
      }
      // entries that the pool could not fill hold nothing
      int64_t none = 0, t;
      const bool have = pg >= 0 && pg < a.n_pages;
      ok = have;
      scan2(none, ok, t, pushed, sums);
      const int64_t s = base + ok - 1;
      if (have) {
        if (s < a.n_pages) a.free_pages[s] = pg;
        else flags |= CG_FLAG_POS_RANGE;  // more pages than the pool has: some came back twice
      }
      base += pushed;
    }
    __syncthreads();
  }
  if (tid == 0) *a.count = int(min(base, int64_t(a.n_pages)));
  if (flags && a.err) atomicOr(a.err, flags);
}

}  // namespace

hipError_t launch_page_map(const int* held, const int* add, int B, const cg_page_pool& pool, int* pages, int max_pages, int P,
                           int N, int* cu, int* lens, int* pos, int* slots, int* err, hipStream_t st) {
  MapArgs a{held, add, B, N, max_pages, P, pool.n_pages, pool.free_pages, pool.free_count, pages, cu, lens, pos, slots, err};
  hipLaunchKernelGGL(map_rows, dim3(1), dim3(kMapThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || N <= kOneLaunch) return e;
  hipLaunchKernelGGL(map_tokens, dim3(unsigned((int64_t(N) + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_release(int* lens, const int* done, int B, const cg_page_pool& pool, int* pages, int max_pages, int P,
                               int* err, bool trim, hipStream_t st) {
  if (B == 0) return hipSuccess;
  MapArgs a{nullptr, nullptr, B, 0, max_pages, P, pool.n_pages, pool.free_pages, pool.free_count, pages, nullptr, lens, nullptr, nullptr, err};
  if (trim) hipLaunchKernelGGL(release_rows<true>, dim3(1), dim3(kMapThreads), 0, st, a, done);
  else hipLaunchKernelGGL(release_rows<false>, dim3(1), dim3(kMapThreads), 0, st, a, done);
  return hipGetLastError();
}

}  // namespace cg
