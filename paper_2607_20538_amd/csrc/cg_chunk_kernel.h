// Attention of a chunk of new tokens over paged, gauge-coded caches: causal, or with a sliding window and
// first positions that stay visible.
//
// Token i of batch row b (n_b new tokens, lens[b] positions held with them) sits at p = lens[b] - n_b + i and
//   o = softmax(scale q Khat^T) Vhat   over t <= p with (window == 0 or t > p - window or t < sinks).
// As in the single-token attention the gauge stays out of the loop over positions: with q' = G_K q and Khat =
// G_K^T zhat^K the scores are q' . zhat^K_t, and o = G_V^T sum_t p_t zhat^V_t, so it is applied once to the
// queries of a tile and once to their sums, on the bf16 matrix cores (split planes of G).
//
// A workgroup takes 128 query rows (tokens x query heads of one KV head) of one batch row and walks their
// visible positions 64 at a time.  The codes of a step become binary16 zhat = fma(q, sc, mn) in LDS once per
// workgroup; both products run on v_mfma_f32_32x32x16_f16 with the queries as columns:
//   S^T = K Q'^T   (lane: one query, half of the 64 positions)  -> softmax without crossing lanes but for one
//                                                                   swap of the halves per step
//   O^T += V^T P^T (the lane's own probabilities are its B operand: the order of the contraction is free, so
//                   V is read in the order that S^T left the positions in, by transposing LDS reads)
// Binary16 and not bf16: codes are exact in both, zhat, q' (scaled by a power of two to at most 2^15) and p then
// carry 11 bits, four times finer than the result's own rounding.  Binary32 results take every operand in
// two binary16 planes (22 bits, three products).  A block's zhat are multiples of 2^-24, binary16's own least step, so
// none is lost below its normal range; the error-free backend's are scaled by a power of two, keys by the largest of
// their step, values by the largest so far, to at most 2^15: binary16 then holds 11 bits down to 2^-29 of it, two planes 22
// bits down to 2^-18 and 2^-40 of it below.  zhat beyond binary16 (the side information allows 2^24), infinities, NaN, and
// error-free values below 2^-29 of the largest make a step "odd": it is summed position by position in binary32, where a
// masked position is left out instead of being multiplied by zero.
//
// Bound by the vector work of decoding and of the exponentials beside the products, which overlap in part (vector
// units busy 50% of the time, matrix cores 34%, two waves per SIMD).  4096 tokens at the end of 20000 positions, 8 KV
// heads x 4, d = 128, 4 bits: 1.78 to 1.91 ms from card to card = 838 to 781 TFLOP/s (a plain
// binary16 matrix product reaches 1169).
#pragma once

#include <type_traits>

#include "cg_internal.h"
#include "cg_device.h"
#include "cg_chunk.h"
#include "cg_chunk_rows.h"
#include "cg_mfma_util.h"

namespace cg {

namespace {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
// Probabilities are kept times 2^6: with a maximum that lags by at most 2^8 they stay below 2^14, and what is
// lost below binary16's subnormals is 2^-31 of the largest.
constexpr float kPBias = 6.0f, kLag = 8.0f;

__device__ __forceinline__ f32x16_t mfma_h(const f16x8_t& a, const f16x8_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pk_h(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), f16x2_t));
}
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_b(float a, float b) {  // bf16 pair, round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
// planes p = 0 .. NP - 1 of a pair: every one the bf16 of what the ones before leave (of an infinity: nothing)
template <int NP>
__device__ __forceinline__ void split_b(float a, float b, uint32_t (&o)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    o[p] = pk_b(a, b);
    a = fabsf(a) < INFINITY ? a - __uint_as_float(o[p] << 16) : 0.0f;
    b = fabsf(b) < INFINITY ? b - __uint_as_float(o[p] & 0xffff0000u) : 0.0f;
  }
}
__device__ __forceinline__ float h_lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w)[0]; }
__device__ __forceinline__ float h_hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w)[1]; }
__device__ __forceinline__ f16x8_t as_f16x8(const u32x4_t& v) { return __builtin_bit_cast(f16x8_t, v); }

// the lane's value and that of the lane 32 away
__device__ __forceinline__ float halves_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// ------------------------------------------------------------------------------------------
// the gauge operands
// ------------------------------------------------------------------------------------------

// Element (row, col) of a head's block-diagonal matrix out of one bf16 plane (G or G^T); zero outside
__device__ __forceinline__ uint32_t gauge_at(const uint16_t* blk, int g, int d, int row, int col) {
  if (row >= d || col >= d) return 0u;
  const int r = row / g;
  if (col / g != r) return 0u;
  return blk[size_t(r) * g * g + size_t(row - r * g) * g + (col - r * g)];
}
// First and last channel of the groups that channels [ch, ch + n) lie in
__device__ __forceinline__ void reached(int g, int ch, int n, int& first, int& last) {
  const float invg = 1.0f / float(g);  // (x + 1/2) / g lies at least 1/512 from an integer
  first = __builtin_amdgcn_readfirstlane(int((float(ch) + 0.5f) * invg)) * g;
  last = __builtin_amdgcn_readfirstlane(int((float(ch + n - 1) + 0.5f) * invg)) * g + g - 1;
}
// Rows row0 .. row0 + ROWS - 1, K-steps kk0 .. kk0 + KS - 1 of NP planes to LDS: row i of plane p at
// (p ROWS + i) (32 KS + 16), its channels in order.  All NT threads of the workgroup.  MOST reads are in flight
// per thread: one at a time they were half of the time of a tile with a window of 1024 positions; eight instead of
// four cost the step loop registers (4096 tokens at 20000 positions 1945 us, 1914 with four).
template <int NP, int ROWS, int KS, int NT, int MOST = 4>
__device__ __forceinline__ void stage_gauge(uint8_t* dst, const uint16_t* const (&planes)[3], size_t gb, int g, int d,
                                            int row0, int kk0) {
  constexpr int PER = 2 * KS, TOTAL = NP * ROWS * PER, ITS = (TOTAL + NT - 1) / NT, UN = ITS < MOST ? ITS : MOST;
  auto plane = [&](int p) { return (p == 0 ? planes[0] : (p == 1 ? planes[1] : planes[2])) + gb; };
  auto put = [&](int p, int i, int gr, const u32x4_t& o) {
    *reinterpret_cast<u32x4_t*>(dst + size_t(p * ROWS + i) * (32 * KS + 16) + 16 * gr) = o;
  };
  if (g % 8) {
#pragma unroll 1
    for (int x = threadIdx.x; x < TOTAL; x += NT) {
      const int p = x / (ROWS * PER), i = x / PER % ROWS, gr = x % PER;
      u32x4_t o = {0u, 0u, 0u, 0u};
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const uint32_t v = gauge_at(plane(p), g, d, row0 + i, 16 * kk0 + 8 * gr + e) << (16 * (e & 1));
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] |= k == e >> 1 ? v : 0u;
      }
      put(p, i, gr, o);
    }
    return;
  }
  const float invg = 1.0f / float(g);  // (x + 1/2) / g lies at least 1/512 from an integer
#pragma unroll 1
  for (int i0 = 0; i0 < ITS; i0 += UN) {
    u32x4_t o[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int x = (i0 + k) * NT + threadIdx.x, p = x / (ROWS * PER), row = row0 + x / PER % ROWS;
      const int c0 = 16 * kk0 + 8 * (x % PER), r = int((float(row) + 0.5f) * invg);
      const bool in = x < TOTAL && row < d && c0 >= r * g && c0 < (r + 1) * g;
      o[k] = u32x4_t{0u, 0u, 0u, 0u};
      if (in) o[k] = *reinterpret_cast<const u32x4_t*>(plane(p) + size_t(r) * g * g + (row - r * g) * g + (c0 - r * g));
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int x = (i0 + k) * NT + threadIdx.x;
      if (x < TOTAL) put(x / (ROWS * PER), x / PER % ROWS, x % PER, o[k]);
    }
  }
}

// ------------------------------------------------------------------------------------------
// codes to binary16
// ------------------------------------------------------------------------------------------

// What a thread holds of 32 neighbouring channels of one position before they go to LDS: the packed words and
// (blocks of whole runs of 32 channels) their side word.
struct Raw32 {
  uint32_t w[8], side;
};

// Stored order of a row: channels 16 kk + 8 half + 4 hc + j sit at 16 kk + 8 hc + 2 j + half, so that the 8
// values a lane half hc takes in K-step kk are one 16-byte granule, its dword j the channels 4 hc + j and
// 8 + 4 hc + j: the pair that one shift of a word holding both codes 16 bits apart selects.

// Codes (kk, hc, j) of a run of 32 channels as the integers of a pair, OR-ed into the bit pattern of (1024, 1024):
// 1024 + q in binary16.  `one` is that pattern and `m` the mask of both codes, held in registers so that
// (x & m) | one is one instruction (it takes no literals).
__device__ __forceinline__ uint32_t code_pair(const uint32_t (&w)[8], int bits, int kk, int hc, int j, uint32_t one, uint32_t m) {
  switch (bits) {
    case 4: {
      const uint32_t u = __builtin_amdgcn_perm(w[2 * kk + 1], w[2 * kk], hc ? 0x07060302u : 0x05040100u);
      return ((u >> (4 * j)) & m) | one;
    }
    case 8:
      return __builtin_amdgcn_perm(w[4 * kk + 2 + hc], w[4 * kk + hc],
                                   uint32_t(j) | 0x0c000c00u | (uint32_t(j + 4) << 16)) | one;
    case 2:
      return ((w[kk] >> (8 * hc + 2 * j)) & m) | one;
    case 3: {  // pairs are 24 bits apart
      const int b = 48 * kk + 12 * hc + 3 * j, o = b >> 5;
      const uint32_t x = __builtin_amdgcn_alignbit(w[o + 1 < 3 ? o + 1 : 2], w[o], b & 31);
      return (x & 7u) | ((x >> 8) & 0x00070000u) | one;
    }
    default: {  // 6 bits: 48 bits apart
      const int b0 = 96 * kk + 24 * hc + 6 * j, b1 = b0 + 48, o0 = b0 >> 5, o1 = b1 >> 5;
      const uint32_t x = __builtin_amdgcn_alignbit(w[o0 + 1 < 6 ? o0 + 1 : 5], w[o0], b0 & 31);
      const uint32_t y = __builtin_amdgcn_alignbit(w[o1 + 1 < 6 ? o1 + 1 : 5], w[o1], b1 & 31);
      return (x & 63u) | ((y & 63u) << 16) | one;
    }
  }
}

// the integer pair (at most 255 each, already under the bits of 1024) as binary16
__device__ __forceinline__ f16x2_t int_pair(uint32_t p) {
  const f16x2_t k = {(_Float16)1024.0f, (_Float16)1024.0f};
  return __builtin_bit_cast(f16x2_t, p) - k;
}

// Four neighbouring channels c .. c + 3 (c a multiple of 4, < d) of a cached position in binary32 (PASS: the error-free
// backend)
template <bool PASS>
__device__ __forceinline__ void load4(const CacheDev& k, const CodecDev& c, size_t row, int d, int ch, float (&out)[4]) {
  if constexpr (PASS) {
    const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(k.codes) + row * d + ch);
    out[0] = v.x; out[1] = v.y; out[2] = v.z; out[3] = v.w;
    return;
  }
  const uint32_t* w = reinterpret_cast<const uint32_t*>(k.codes) + row * size_t(d * c.bits / 32);
  const int bit = ch * c.bits, o = bit >> 5, last = d * c.bits / 32 - 1;
  const uint64_t v = ((uint64_t(w[min(o + 1, last)]) << 32) | w[o]) >> (bit & 31);
  const uint32_t s = k.side[row * size_t(d / c.n) + ch / c.n];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    out[e] = dequantize(uint32_t(v >> (c.bits * e)) & ((1u << c.bits) - 1u), f16_bits_to_f32(s & 0xffffu), f16_bits_to_f32(s >> 16));
}

// ------------------------------------------------------------------------------------------
// the kernel
// ------------------------------------------------------------------------------------------
// D: channels of a row rounded up (zeros past d); PL: binary16 planes of an operand.
// Always four waves, also where the queries fill one: the others decode its codes.  32 rows of one token, 8 KV heads
// x 4, d = 128, n = 32, up to 8000 positions: 463 us with one wave, 297 with two, 146 with four.
constexpr int NW = kChunkWaves;
// BITS: the code width of rows that decode in whole runs (chunk_wide; 0: any width, read at run time), or
// kAnyLayout: any block and row width, or kErrorFree: the error-free backend, four channels at a time.  A width known to the
// compiler took 2088 -> 1850 us (4096 tokens at 20000 positions, 4 bits): the branches over widths, twice a step, and
// the registers of all of them.
constexpr int kAnyLayout = -1, kErrorFree = -2;
constexpr int kFillOps = 11;  // vector instructions of the next step's codes beside each product of the scores

template <int D, int PL>
struct ChunkShape {
  static constexpr int KP = 2 * D + 16;                          // bytes between K rows: an odd number of granules
  static constexpr int VP = 2 * D + (D % 64 == 32 ? 0 : 64);     // V rows: 4 of them cover all banks once (64 mod 128)
  static constexpr int plane = kStep * (KP + VP);
  static constexpr int buffers = PL == 1 && D <= 128 ? 2 : 1;
  static constexpr int bytes = plane * PL * buffers;
  static constexpr int all = bytes + 128;                        // with the waves' flags and maxima
  static_assert(VP % 64 == 0 && kStep * KP % 64 == 0, "V runs on multiples of 64 bytes");
};

template <int D, int PL, int BITS>
__global__ __launch_bounds__(64 * NW, D <= 128 && PL == 1 ? 2 : 1) void chunk_attend(ChunkDev a, GaugeDev G, CodecDev c) {
  using SH = ChunkShape<D, PL>;
  constexpr bool WIDE = BITS >= 0, PASS = BITS == kErrorFree;
  const int bits = BITS > 0 ? BITS : c.bits;
  constexpr int NT = 64 * NW, KK = D / 16, CT = D / 32, RUNS = D / 32;
  constexpr int ITEMS = 2 * kStep * RUNS, IT = (ITEMS + NT - 1) / NT;  // (position, run) of K, then of V
  static_assert(ITEMS % NT == 0, "items per thread");
  extern __shared__ __attribute__((aligned(64))) uint8_t sm[];
  uint32_t(*state)[NW] = reinterpret_cast<uint32_t(*)[NW]>(sm + SH::bytes);  // per step parity and wave: whether its items make the step odd
  float(*most)[2][NW] = reinterpret_cast<float(*)[2][NW]>(sm + SH::bytes + 32);  // PASS: the largest of its keys, of its values

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hc = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = a.kc.H, d = a.q.d, inner = H * a.nqc;
  int bid = blockIdx.x;
  const int hq = bid % inner;
  bid /= inner;
  const int sp = bid % a.nsplit;
  bid /= a.nsplit;
  const int tile = bid % a.ntile, lv = bid / a.ntile;
  const int h = hq / a.nqc, qc = hq - h * a.nqc, l = lv + a.l0;
  if (blockIdx.x == 0 && a.err) {  // rows that cannot be taken
    for (int b = tid; b < a.B; b += NT) {
      int c0;
      if (row_tokens(a, b, c0) < 0) atomicOr(a.err, CG_FLAG_POS_RANGE);
    }
  }
  const QTile qt = find_tile(a, tile);
  if (qt.b < 0) return;
  const int ntok = min(a.tq, qt.n - qt.i0);
  const int j0 = qc * a.heads, nh = min(a.heads, a.grp - j0), rows = ntok * nh;
  int held = a.lens[qt.b];
  const bool bad_row = held < qt.n || held > a.cap;
  if (bad_row) {
    if (tid == 0 && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
    held = 0;
  }
  const int pa = held - qt.n + qt.i0, pb = pa + ntok - 1;  // positions of the tile's tokens
  // steps: those that hold sinks before the window, then from the window's first position to the last token
  int lo_t = 0, sink_t = 0, nstep = 0;
  if (!bad_row) {
    if (a.window > 0) {
      lo_t = max(0, pa - a.window + 1) / kStep;
      sink_t = min((min(a.sinks, pb + 1) + kStep - 1) / kStep, lo_t);
    }
    nstep = sink_t + pb / kStep - lo_t + 1;
  }
  const int per = (nstep + a.nsplit - 1) / a.nsplit, v0 = min(nstep, sp * per), v1 = min(nstep, v0 + per);
  auto step_pos = [&](int v) { return kStep * (v < sink_t ? v : lo_t + v - sink_t); };

  // this lane's query (columns past the tile repeat its last one and are not stored)
  const int r = min(32 * w + n, rows - 1);
  const int tok = r / nh, jj = r - tok * nh;
  const int pq = pa + tok;
  const int plow = a.window > 0 ? max(pq - a.window, -1) : -1;   // positions up to here are hidden unless a sink
  // the first and last position of the wave's queries
  const int wlo = pa + min(32 * w, rows - 1) / nh, whi = pa + min(32 * w + 31, rows - 1) / nh;
  const bool idle = 32 * w >= rows;                     // a wave without queries only moves codes and gauges
  const size_t qoff = size_t(lv) * a.q.sl + size_t(h * a.grp + j0 + jj) * a.q.sh + size_t(qt.tok0 + qt.i0 + tok) * a.q.st;

  // ---- loads of a step: page, then this thread's runs
  constexpr bool AHEAD = WIDE && IT * D <= 256;  // a step's codes wait in registers while the step before is computed
  Raw32 raw[AHEAD ? IT : 1] = {};
  size_t srow = 0;       // cache row of the step's first position
  bool have = false;     // the step's page is inside the pool
  constexpr bool KEEP = PASS && IT <= 2;
  int up[2] = {0, 200};  // PASS: exponents that the step's keys and the values so far are scaled by (200: no values yet)
  const int words = d * bits / 32, nblk = WIDE ? d / c.n : 1;  // words and side words of a row
  auto item = [&](int i, bool& val, int& pos, int& run) {
    // the same side for a whole wave
    const int x0 = (ITEMS / 2) % NT == 0 ? i * NT : i * NT + 64 * w;
    val = x0 >= ITEMS / 2;
    const int y = ((ITEMS / 2) % NT == 0 ? i * NT + tid : x0 + lane) - (val ? ITEMS / 2 : 0);
    pos = y / RUNS;
    run = y % RUNS;
  };
  // Buffer loads: the step's rows are the buffer, in scalar registers, and a thread keeps a 32-bit offset (as
  // 64-bit addresses the offsets took registers enough to spill)
  auto rows_at = [&](const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, kStep * bytes, 0x00027000);
  };
  auto load_run = [&](Raw32& o, int i) {
    bool val;
    int pos, run;
    item(i, val, pos, run);
    // a base that the workgroup shares and an offset that the thread keeps
    const CacheDev& k = val ? a.vc : a.kc;
    const auto rows = rows_at(k.codes + srow * (4 * words), 4 * words);
    // (channels past the row: offsets past the buffer, which read as zeros)
    const bool none = 32 * run >= d;
    const int at = none ? kStep * 4 * words : 4 * (pos * words + run * bits);
    auto words_at = [&](auto width, int i0) {  // `width` words from word i0 on, in one load
      constexpr int W = decltype(width)::value;
      uint32_t u[W];
      if constexpr (W == 2) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(rows, at + 4 * i0, 0, 0);
        u[0] = x[0], u[1] = x[1];
      } else if constexpr (W == 3) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b96(rows, at + 4 * i0, 0, 0);
        u[0] = x[0], u[1] = x[1], u[2] = x[2];
      } else {
        const auto x = __builtin_amdgcn_raw_buffer_load_b128(rows, at + 4 * i0, 0, 0);
        u[0] = x[0], u[1] = x[1], u[2] = x[2], u[3] = x[3];
      }
#pragma unroll
      for (int e = 0; e < W; ++e) o.w[i0 + e] = u[e];
    };
    switch (bits) {  // rows of whole runs: every run starts on a multiple of its load's width
      case 4: words_at(std::integral_constant<int, 4>(), 0); break;
      case 8:
        words_at(std::integral_constant<int, 4>(), 0);
        words_at(std::integral_constant<int, 4>(), 4);
        break;
      case 2: words_at(std::integral_constant<int, 2>(), 0); break;
      case 3: words_at(std::integral_constant<int, 3>(), 0); break;
      default:
        words_at(std::integral_constant<int, 2>(), 0);
        words_at(std::integral_constant<int, 2>(), 2);
        words_at(std::integral_constant<int, 2>(), 4);
    }
    o.side = __builtin_amdgcn_raw_buffer_load_b32(rows_at(k.side + srow * nblk, 4 * nblk), none ? kStep * 4 * nblk : 4 * (pos * nblk + 32 * run / c.n), 0, 0);
  };
  // pages are looked up a step ahead of the fetch; the next look: step, page of the row, position in it
  const int* table = a.pt.pages + size_t(qt.b) * a.pt.max_pages;
  const int P = a.pt.page_size;
  const size_t row0 = (size_t(l) * a.kc.B * H + h) * P, prows = size_t(H) * P;
  int look_v = v0, look_p = step_pos(v0) / P, look_off = step_pos(v0) - look_p * P;
  int page = -1, off = 0;
  auto look = [&]() {
    page = look_v < v1 ? table[look_p] : -1;
    off = look_off;
    look_off += kStep;
    if (look_off >= P) {
      look_off = 0;
      ++look_p;
    }
    if (++look_v == sink_t) {  // from the sinks to the window
      look_p = kStep * lo_t / P;
      look_off = kStep * lo_t - look_p * P;
    }
  };
  look();
  auto fetch = [&]() {
    const int pg = __builtin_amdgcn_readfirstlane(page), at = off;
    look();
    have = pg >= 0 && pg < a.kc.B;
    if (!have) {
      if (tid == 0 && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
      return;
    }
    srow = row0 + size_t(pg) * prows + at;
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < IT; ++i) load_run(raw[i], i);
    }
  };
  // codes -> binary16 rows in LDS; positions from `held` on become zeros (their bytes may hold anything)
  // decode() gives the granules of item i to out(i, plane, 2 kk + half, granule), store() puts one into a buffer.
  auto store = [&](uint8_t* buf, int i, int plane, int g, const u32x4_t& o) {
    bool val;
    int pos, run;
    item(i, val, pos, run);
    // V rows that share their banks (every fourth) keep the granules of a run in another order; their runs
    // start on multiples of 64 bytes, so granule g of one is at its first one's address ^ 16 g
    const uint32_t dst = uint32_t(buf - sm) + 64 * run + (val ? kStep * SH::KP + pos * SH::VP + 16 * (pos & 3) : pos * SH::KP);
    *reinterpret_cast<u32x4_t*>(sm + (val ? dst ^ (16 * g) : dst + 16 * g) + plane * SH::plane) = o;
  };
  auto decode = [&](int v, auto out) {
    const int t0 = step_pos(v);
    bool st = false;  // zhat that binary16 does not hold
    float zp[KEEP ? IT : 1][8][4];  // PASS: this thread's values
    if constexpr (PASS) {
      // the largest finite magnitudes of the step first, its values kept where registers last (32 single tokens of up
      // to 8000 positions, 8 KV heads x 4, bf16 results: d = 128 594 us kept, 997 read twice; d = 256 3283 and 2551)
      float mx[2] = {0.0f, 0.0f};
      auto largest = [&](const float (&z)[8][4], bool val) {
        float m = 0.0f;
#pragma unroll
        for (int g = 0; g < 8; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = fabsf(z[g][e]);
            if (x < INFINITY) m = fmaxf(m, x);
            else st = true;
          }
        (val ? mx[1] : mx[0]) = fmaxf(val ? mx[1] : mx[0], m);
      };
      auto read = [&](float (&z)[8][4], int i, bool& val) {
        int pos, run;
        item(i, val, pos, run);
        const bool live = have && t0 + pos < held;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const int ch = 32 * run + 4 * g;
#pragma unroll
          for (int e = 0; e < 4; ++e) z[g][e] = 0.0f;
          if (live && ch < d) load4<PASS>(val ? a.vc : a.kc, c, srow + pos, d, ch, z[g]);
        }
      };
      if constexpr (KEEP) {
        bool side[IT];
#pragma unroll
        for (int i = 0; i < IT; ++i) read(zp[i], i, side[i]);
#pragma unroll
        for (int i = 0; i < IT; ++i) largest(zp[i], side[i]);
      } else {
#pragma unroll 1
        for (int i = 0; i < IT; ++i) {
          bool val;
          read(zp[0], i, val);
          largest(zp[0], val);
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx[s] = fmaxf(mx[s], __shfl_xor(mx[s], o));
        if (lane == 0) most[v & 1][s][w] = mx[s];
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float m = most[v & 1][s][0];
#pragma unroll
        for (int i = 1; i < NW; ++i) m = fmaxf(m, most[v & 1][s][i]);
        const int e = m > 0.0f ? 15 - __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(m)) : 200;
        up[s] = s ? min(up[s], e) : e;
      }
    }
    auto one = [&](int i, Raw32& rw) {
      bool val;
      int pos, run;
      item(i, val, pos, run);
      const bool live = have && t0 + pos < held;  // (nothing of a page outside the pool)
      auto put = [&](int plane, int kk, int half, const u32x4_t& o) { out(i, plane, 2 * kk + half, o); };
      // the pair (codes p) of a granule with its two blocks' side words
      auto pair = [&](uint32_t p, f16x2_t sc, f16x2_t mn, uint32_t& hi, uint32_t& lo) {
        const f16x2_t q = int_pair(p);
        if constexpr (PL == 1) {
          hi = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(q, sc, mn));
        } else {
          const float z0 = fmaf((float)q[0], (float)sc[0], (float)mn[0]), z1 = fmaf((float)q[1], (float)sc[1], (float)mn[1]);
          hi = pk_h(z0, z1);
          lo = pk_h(z0 - h_lo(hi), z1 - h_hi(hi));
        }
      };
      if constexpr (WIDE) {
        const uint32_t s = live ? rw.side : 0u;
        const float mnf = f16_bits_to_f32(s & 0xffffu), top = fmaf(float((1 << bits) - 1), f16_bits_to_f32(s >> 16), mnf);
        if (!(fabsf(top) <= 65504.0f && fabsf(mnf) <= 65504.0f)) st = true;
        const _Float16 m1 = __builtin_bit_cast(_Float16, uint16_t(s)), s1 = __builtin_bit_cast(_Float16, uint16_t(s >> 16));
        const f16x2_t mn = {m1, m1}, sc = {s1, s1};
        auto all = [&](auto width) {
          uint32_t one = 0x64006400u, m = ((1u << decltype(width)::value) - 1u) * 0x00010001u;
          asm("" : "+v"(one), "+v"(m));
#pragma unroll
          for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              u32x4_t hi, lo;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t x, y = 0;
                pair(code_pair(rw.w, decltype(width)::value, kk, half, j, one, m), sc, mn, x, y);
                hi[j] = x;
                lo[j] = y;
              }
              put(0, kk, half, hi);
              if constexpr (PL == 2) put(1, kk, half, lo);
            }
        };
        switch (bits) {
          case 4: all(std::integral_constant<int, 4>()); break;
          case 8: all(std::integral_constant<int, 8>()); break;
          case 2: all(std::integral_constant<int, 2>()); break;
          case 3: all(std::integral_constant<int, 3>()); break;
          default: all(std::integral_constant<int, 6>()); break;
        }
      } else {
        // any block width and row width, or the error-free backend: four channels at a time in binary32
        auto granule = [&](int g4) {
          float z[2][4];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int ch = 32 * run + 16 * (g4 >> 1) + 8 * q + 4 * (g4 & 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[q][e] = 0.0f;
            if constexpr (KEEP) {
#pragma unroll
              for (int e = 0; e < 4; ++e) z[q][e] = zp[i][4 * (g4 >> 1) + 2 * q + (g4 & 1)][e];
            } else {
              if (live && ch < d) load4<PASS>(val ? a.vc : a.kc, c, srow + pos, d, ch, z[q]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool any = z[q][e] != 0.0f;
              if constexpr (PASS) z[q][e] = __builtin_amdgcn_ldexpf(z[q][e], up[val]);
              const float m = fabsf(z[q][e]);
              if (!(m <= 65504.0f) || (PASS && any && m < 0x1p-14f)) st = true;
            }
          }
          u32x4_t hi, lo;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            hi[j] = pk_h(z[0][j], z[1][j]);
            lo[j] = pk_h(z[0][j] - h_lo(hi[j]), z[1][j] - h_hi(hi[j]));
          }
          put(0, g4 >> 1, g4 & 1, hi);
          if constexpr (PL == 2) put(1, g4 >> 1, g4 & 1, lo);
        };
        if constexpr (KEEP) {
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) granule(g4);
        } else {
#pragma unroll 1
          for (int g4 = 0; g4 < 4; ++g4) granule(g4);
        }
      }
    };
    if constexpr (AHEAD || KEEP) {
#pragma unroll
      for (int i = 0; i < IT; ++i) one(i, raw[AHEAD ? i : 0]);
    } else {
#pragma unroll 1
      for (int i = 0; i < IT; ++i) {
        if constexpr (WIDE) load_run(raw[0], i);
        one(i, raw[0]);
      }
    }
    return __builtin_amdgcn_ballot_w64(st) ? 1u : 0u;  // (in any lane of the wave)
  };
  auto fill = [&](int v, uint8_t* buf) {
    state[v & 1][w] = decode(v, [&](int i, int plane, int g, const u32x4_t& o) { store(buf, i, plane, g, o); });
  };

  if (v0 < v1) fetch();

  // ---- the queries: q' = G_K q for this lane's column, binary16 B operands
  f16x8_t Q[PL][KK];
  float cs = 0.0f;  // score = S cs, in powers of two
  {
    f32x16_t z[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) z[ct] = f32x16_t{};
    const size_t gb = ((size_t(l) * 2 + 0) * G.H + h) * G.R * size_t(G.g) * G.g;
    // The gauge in one pass where LDS holds it, here and at the end, and the queries two K-steps ahead of their
    // products: in passes of 64 channels (32 at the end) with every query waited for, 3 rows of 37 tokens took 34 us
    // (29 so), 6000 tokens behind a window of 64 positions 124 (116).
    constexpr int GP = PL == 1 ? 2 : 3, KQ = 2;
    constexpr int KC = GP * D * (32 * KK + 16) <= SH::bytes ? KK : (D == 256 && PL == 1 ? 2 : 4), GPITCH = 32 * KC + 16;
    static_assert(GP * D * GPITCH <= SH::bytes, "space of the gauge");
    const bool qb = a.q.bf16;
    u32x4_t xq[KQ];  // bf16 queries of the KQ K-steps that come next
    auto read_q = [&](int kk0) {
#pragma unroll
      for (int i = 0; i < KQ; ++i) {
        const int ch = 16 * (kk0 + i) + 8 * hc;
        xq[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (qb && ch < d) xq[i] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.q.ptr) + qoff + ch);
      }
    };
    // one K-step: NX planes of its queries
    auto kstep = [&](int kk, int k0, const auto& x, auto nx) {
      constexpr int NX = decltype(nx)::value;
      const uint8_t* src = sm + n * GPITCH + 32 * (kk - k0) + 16 * hc;
      int c0, c1;
      reached(G.g, 16 * kk, 16, c0, c1);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        if (32 * ct > c1 || 32 * ct + 31 < c0) continue;  // no group of the K-step reaches this channel tile
        bf16x8_t A[GP];
#pragma unroll
        for (int p = 0; p < GP; ++p) A[p] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(src + (p * D + 32 * ct) * GPITCH));
#pragma unroll
        for (int s = 0; s < NX; ++s)
#pragma unroll
          for (int p = 0; p < GP; ++p)
            if (p + s < 3) z[ct] = mfma(A[p], as_bf16x8(x[s]), z[ct]);
      }
    };
    read_q(0);
    for (int k0 = 0; 16 * k0 < d; k0 += KC) {
      if (k0) __syncthreads();
      stage_gauge<GP, D, KC, NT>(sm, G.hi, gb, G.g, d, 0, k0);
      __syncthreads();
      if (qb) {
#pragma unroll 1
        for (int k4 = k0; k4 < k0 + KC && 16 * k4 < d; k4 += KQ) {
          u32x4_t xc[KQ];
#pragma unroll
          for (int i = 0; i < KQ; ++i) xc[i] = xq[i];
          read_q(k4 + KQ);
#pragma unroll
          for (int i = 0; i < KQ; ++i) {
            const u32x4_t one[1] = {xc[i]};
            if (16 * (k4 + i) < d) kstep(k4 + i, k0, one, std::integral_constant<int, 1>());
          }
        }
        continue;
      }
#pragma unroll 1
      for (int kk = k0; kk < k0 + KC && 16 * kk < d; ++kk) {
        const int ch = 16 * kk + 8 * hc;
        u32x4_t x[3];
#pragma unroll
        for (int p = 0; p < 3; ++p) x[p] = u32x4_t{0u, 0u, 0u, 0u};
        if (ch < d) {
          const float* src = static_cast<const float*>(a.q.ptr) + qoff + ch;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t o[3];
            split_b<3>(src[2 * e], src[2 * e + 1], o);
#pragma unroll
            for (int p = 0; p < 3; ++p) x[p][e] = o[p];
          }
        }
        kstep(kk, k0, x, std::integral_constant<int, 3>());
      }
    }
    __syncthreads();  // the gauge is read
    float mx = 0.0f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fabsf(z[ct][e]));
    mx = halves_max(mx);
    const int ex = mx > 0.0f && mx < INFINITY ? __builtin_amdgcn_frexp_expf(mx) : 0;
    const float sign = a.scale < 0.0f ? -1.0f : (a.scale > 0.0f ? 1.0f : 0.0f);
    // the largest to [2^14, 2^15), as binary16's least step would otherwise take bits from the small ones
    cs = a.scale == 0.0f ? 1.0f : fmaxf(__builtin_amdgcn_ldexpf(fabsf(a.scale) * kLog2e, ex - 15), 1e-37f);  // (not 0: 0 times a hidden score)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      u32x4_t hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x0 = sign * __builtin_amdgcn_ldexpf(z[kk >> 1][8 * (kk & 1) + j], 15 - ex);
        const float x1 = sign * __builtin_amdgcn_ldexpf(z[kk >> 1][8 * (kk & 1) + 4 + j], 15 - ex);
        hi[j] = pk_h(x0, x1);
        lo[j] = pk_h(x0 - h_lo(hi[j]), x1 - h_hi(hi[j]));
      }
      Q[0][kk] = as_f16x8(hi);
      if constexpr (PL == 2) Q[PL - 1][kk] = as_f16x8(lo);
    }
  }

  f32x16_t O[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) O[ct] = f32x16_t{};
  float m = -INFINITY, lsum = 0.0f;  // running maximum (in S) and this lane half's sum

  // ---- steps
  // FUSED: with two buffers the next step's codes are decoded while this one's scores are on the matrix cores (16
  // products leave room for about ten vector instructions each), with one barrier a step; else before them.
  // The body is one path whatever the step: where it is not, the sums are moved between registers in every step (64
  // moves of a wave's 340 vector instructions).  So an odd step leaves the loop, which is entered again after it, and a step that
  // a wave sees nothing of runs with every weight 0; a wave without queries has a loop of its own.
  constexpr bool FUSED = AHEAD && SH::buffers == 2;
  auto buf_of = [&](int v) { return sm + (SH::buffers == 2 ? (v & 1) * SH::plane * PL : 0); };
  int v = v0;
  size_t crow = 0;    // cache row of step v's first position
  bool ok = false;    // its page is inside the pool
  bool skip = false;  // (FUSED) the odd step v is summed: what is left of it is to decode the next one's codes
  auto advance = [&]() {  // what was fetched is step v, the one after it is fetched
    ok = have;
    crow = srow;
  };
  if (FUSED && v < v1) {
    advance();
    fill(v, buf_of(v));
    if (v + 1 < v1) fetch();
    __syncthreads();
  }
  // whether step v, in its buffer, is odd
  auto odd_step = [&]() {
    uint32_t st = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) st |= state[v & 1][i];
    return ok && !skip && __builtin_amdgcn_readfirstlane(st);
  };
  // An odd step: its positions in binary32, 16 of K and V at a time through its buffer (in the lanes' order: the
  // values of (kk, hc) at 16 kk + 8 hc, for V of (ct, i, hc) at 32 ct + 8 i + 4 hc), each given to `take`
  auto odd_rows = [&](auto take) {
    constexpr int SUB = 16;
    static_assert(2 * SUB * D * 4 <= SH::plane * PL, "space of the rows");
    float* rows32 = reinterpret_cast<float*>(buf_of(v));
    const int live = min(kStep, held - step_pos(v));
#pragma unroll 1
    for (int s0 = 0; s0 < live; s0 += SUB) {
      __syncthreads();
#pragma unroll 1
      for (int x = tid; x < 2 * SUB * (D / 4); x += NT) {
        const bool val = x >= SUB * (D / 4);
        const int y = val ? x - SUB * (D / 4) : x, pos = y / (D / 4), ch = 4 * (y - pos * (D / 4));
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (s0 + pos < live && ch < d) load4<PASS>(val ? a.vc : a.kc, c, crow + s0 + pos, d, ch, z);
        if constexpr (PASS) {
          if (val) {
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = __builtin_amdgcn_ldexpf(z[e], up[1]);
          }
        }
        float* dst = rows32 + (val ? SUB * D : 0) + pos * D + (ch & ~15);
        const int half = (ch >> 3) & 1, h4 = (ch >> 2) & 1;  // channels 16 kk + 8 half + 4 h4 ..
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[8 * h4 + 2 * j + half] = z[j];
      }
      __syncthreads();
      take(s0, min(SUB, live - s0), rows32 + 8 * hc, rows32 + SUB * D + 4 * hc);
    }
    if constexpr (FUSED) {
      // the step's products are formed once more, with weights 0: of zeros
      __syncthreads();
      for (int x = tid; x < SH::plane / 16; x += NT) reinterpret_cast<u32x4_t*>(rows32)[x] = u32x4_t{0u, 0u, 0u, 0u};
      __syncthreads();
      skip = true;
    } else {
      ++v;
    }
  };
  // the start of a step that is not FUSED
  auto begin = [&]() {
    advance();
    if (SH::buffers == 1 && v > v0) __syncthreads();  // the step before is read
    fill(v, buf_of(v));
    if (v + 1 < v1) fetch();
    __syncthreads();
  };
  // the end of the scores of a FUSED one
  auto turn = [&]() {
    advance();
    if (v + 2 < v1) fetch();
  };
  if (idle) {
    while (v < v1) {
      if constexpr (!FUSED) begin();
      if (odd_step()) {
        odd_rows([](int, int, const float*, const float*) {});
        continue;
      }
      skip = false;
      if constexpr (FUSED) {
        fill(v + 1, buf_of(v + 1));
        turn();
        __syncthreads();
      }
      ++v;
    }
  }
  while (v < v1) {
    bool odd = false;
    for (; v < v1; ++v) {
      const int t0 = step_pos(v);
      const uint8_t* buf = buf_of(v);
      const int was = up[1];
      if constexpr (!FUSED) begin();
      if constexpr (PASS) {
        if (up[1] != was) {  // (O is zero where there were no values)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) O[ct][e] = __builtin_amdgcn_ldexpf(O[ct][e], up[1] - was);
        }
      }
      odd = odd_step();
      if (odd) break;
      // nothing of the step is visible to this wave's queries, or it holds nothing
      const bool blank = !ok || skip;
      skip = false;
      // scores; operands KB K-steps ahead of the products
      f32x16_t S[2];
      S[0] = f32x16_t{};
      S[1] = f32x16_t{};
      constexpr int KB = FUSED ? 1 : 2;
      const uint8_t* kb = buf + n * SH::KP + 16 * hc;
      f16x8_t kf[2][KB][2][PL];  // buffer, K-step, positions, plane
      auto kload = [&](int s, int k2) {
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int ps = 0; ps < 2; ++ps)
#pragma unroll
            for (int p = 0; p < PL; ++p)
              kf[s][i][ps][p] = as_f16x8(*reinterpret_cast<const u32x4_t*>(kb + 32 * ps * SH::KP + 32 * (KB * k2 + i) + p * SH::plane));
      };
      __builtin_amdgcn_sched_barrier(0);
      kload(0, 0);
#pragma unroll
      for (int k2 = 0; k2 < KK / KB; ++k2) {
        if (k2 + 1 < KK / KB) kload((k2 + 1) & 1, k2 + 1);
        if constexpr (!FUSED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int ps = 0; ps < 2; ++ps) {
            const int kk = KB * k2 + i;
            S[ps] = mfma_h(kf[k2 & 1][i][ps][0], Q[0][kk], S[ps]);
            if constexpr (PL == 2) {
              S[ps] = mfma_h(kf[k2 & 1][i][ps][0], Q[PL - 1][kk], S[ps]);
              S[ps] = mfma_h(kf[k2 & 1][i][ps][PL - 1], Q[0][kk], S[ps]);
            }
          }
        if constexpr (!FUSED) __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (FUSED) {
        // the next step's codes, between the products; past all of this one's reads they go to the other buffer
        // (past the last step what is written there is not read)
        u32x4_t dec[IT][4];
        const uint32_t flags = decode(v + 1, [&](int i, int, int g, const u32x4_t& o) { dec[i][g] = o; });
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
        for (int k2 = 0; k2 < KK; ++k2) {
          if (k2 + 1 < KK) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, kFillOps, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) store(buf_of(v + 1), i, 0, g, dec[i][g]);
        state[(v + 1) & 1][w] = flags;
        turn();
      }
      if constexpr (PASS) {
#pragma unroll
        for (int ps = 0; ps < 2; ++ps)
#pragma unroll
          for (int e = 0; e < 16; ++e) S[ps][e] = __builtin_amdgcn_ldexpf(S[ps][e], -up[0]);
      }
      // hidden positions: after the lane's token, or before its window and no sink
      const bool whole = !blank && t0 + kStep - 1 <= wlo && (a.window == 0 || t0 > whi - a.window || t0 + kStep <= a.sinks);
      if (!whole) {
        // bit c: position t0 + 4 hc + c is seen; element (ps, e) is bit 32 ps + 8 (e / 4) + e % 4
        const int t1 = t0 + 4 * hc;
        auto below = [](int x) { return x <= 0 ? 0ull : (x >= 64 ? ~0ull : (1ull << x) - 1ull); };
        const uint64_t seen = blank ? 0ull : below(pq - t1 + 1) & (~below(plow - t1 + 1) | below(a.sinks - t1));
        const uint32_t half[2] = {uint32_t(seen), uint32_t(seen >> 32)};
#pragma unroll
        for (int ps = 0; ps < 2; ++ps)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t keep = uint32_t(__builtin_amdgcn_sbfe(int(half[ps]), 8 * (e >> 2) + (e & 3), 1));
            S[ps][e] = __uint_as_float((__float_as_uint(S[ps][e]) & keep) | (0xff800000u & ~keep));
          }
      }
      float mx = S[0][0];
#pragma unroll
      for (int ps = 0; ps < 2; ++ps)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, S[ps][e]);
      mx = halves_max(mx);
      // the maximum moves only when a score passes it by 2^kLag: the sums are seldom rescaled
      const bool lift = mx > m && (m == -INFINITY || (mx - m) * cs > kLag);
      if (__builtin_amdgcn_ballot_w64(lift)) {
        const float mn = fmaxf(m, mx);
        const float al = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - mn) * cs);
        m = mn;
        lsum *= al;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int e = 0; e < 16; ++e) O[ct][e] *= al;
      }
      const float off = kPBias - (m == -INFINITY ? 0.0f : m * cs);
      float ls[2] = {0.0f, 0.0f};
      // values: element e of the lane's operand is position 16 kp + 8 (e / 4) + 4 hc + e % 4
      const uint8_t* vb = buf + kStep * SH::KP + (4 * hc + ((lane >> 2) & 3)) * SH::VP +
                          16 * ((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ ((lane >> 2) & 3)) + 8 * (lane & 1);
      auto vfrag = [&](int plane, int ct, int kp) {
        typedef __attribute__((address_space(3))) s16x4_t* lds4;
        const uint8_t* src = vb + plane * SH::plane + 16 * kp * SH::VP + 64 * ct;
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(src));
        const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(src + 8 * SH::VP));
        return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      // probabilities of K-step kp, operands in P
      f16x8_t P[2][PL];
      auto weights = [&](int s, int kp) {
        u32x4_t hi, lo;
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) {
          const int e = 8 * (kp & 1) + 2 * e2;
          const float p0 = __builtin_amdgcn_exp2f(fmaf(S[kp >> 1][e], cs, off));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(S[kp >> 1][e + 1], cs, off));
          const uint32_t both = pk_h(p0, p1);
          hi[e2] = both;
          if constexpr (PL == 2) {
            ls[0] += p0;
            ls[1] += p1;
            lo[e2] = pk_h(p0 - h_lo(both), p1 - h_hi(both));
          } else {
            // the rounded weights, as the values meet them (v_dot2_f32_f16 adds both to binary32 exactly)
            const f16x2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
            ls[e2 & 1] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, both), ones, ls[e2 & 1], false);
          }
        }
        P[s][0] = as_f16x8(hi);
        if constexpr (PL == 2) P[s][PL - 1] = as_f16x8(lo);
      };
      // the products of K-step kp run while the probabilities of the next are computed
      constexpr int CB = CT < 4 ? CT : 4;  // channel tiles whose operands are loaded together
      f16x8_t vf[2][CB][PL];
      auto vload = [&](int s, int x) {  // batch x: K-step x / (CT / CB), channel tiles CB (x % (CT / CB)) ..
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
          for (int p = 0; p < PL; ++p) vf[s][i][p] = vfrag(p, CB * (x % (CT / CB)) + i, x / (CT / CB));
      };
      constexpr int NB = 4 * (CT / CB);
      vload(0, 0);
      weights(0, 0);
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const int kp = x / (CT / CB), c0 = CB * (x % (CT / CB));
        if (x + 1 < NB) vload((x + 1) & 1, x + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < CB; ++i) {
          O[c0 + i] = mfma_h(vf[x & 1][i][0], P[kp & 1][0], O[c0 + i]);
          if constexpr (PL == 2) {
            O[c0 + i] = mfma_h(vf[x & 1][i][0], P[kp & 1][PL - 1], O[c0 + i]);
            O[c0 + i] = mfma_h(vf[x & 1][i][PL - 1], P[kp & 1][0], O[c0 + i]);
          }
        }
        if (c0 == 0 && kp + 1 < 4) weights((kp + 1) & 1, kp + 1);
        if (x + 1 < NB) {
#pragma unroll
          for (int i = 0; i < CB * (PL == 2 ? 3 : 1); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, 9, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      lsum += ls[0] + ls[1];
      if constexpr (FUSED) __syncthreads();
    }
    if (!odd) break;
    {
      const int t0 = step_pos(v);
      odd_rows([&](int s0, int count, const float* krows, const float* vrows) {
#pragma unroll 1
        for (int u = 0; u < count; ++u) {
          const float* kr = krows + u * D;
          const float* vr = vrows + u * D;
          const int t = t0 + s0 + u;
          const bool seen = t <= pq && (t > plow || t < a.sinks);
          float s = 0.0f;
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            // (opaque: the queries in binary32 would otherwise be kept for this rare path, in registers
            // that the others need)
            u32x4_t qa = __builtin_bit_cast(u32x4_t, Q[0][kk]), qb = __builtin_bit_cast(u32x4_t, Q[PL - 1][kk]);
            asm volatile("" : "+v"(qa), "+v"(qb));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float q = (e & 1) ? h_hi(qa[e >> 1]) : h_lo(qa[e >> 1]);
              if constexpr (PL == 2) q += (e & 1) ? h_hi(qb[e >> 1]) : h_lo(qb[e >> 1]);
              s = fmaf(q, kr[16 * kk + e], s);
            }
          }
          s = halves_sum(s);
          const float mn = seen ? fmaxf(m, s) : m;
          const float al = m == mn ? 1.0f : __builtin_amdgcn_exp2f((m - mn) * cs);
          const float p = seen ? __builtin_amdgcn_exp2f(fmaf(s, cs, kPBias - (mn == -INFINITY ? 0.0f : mn * cs))) : 0.0f;
          m = mn;
          lsum = fmaf(lsum, al, hc ? 0.0f : p);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float o = O[ct][e] * al;
              O[ct][e] = seen ? fmaf(p, vr[32 * ct + 8 * (e >> 2) + (e & 3)], o) : o;
            }
        }
      });
    }
  }
  // ---- o = G_V^T (sums / normaliser): the sums are the B operand as they lie
  const float lall = halves_sum(lsum), inv = lall == 0.0f ? 0.0f : 1.0f / lall;  // nothing visible: zeros
  constexpr int OP = PL == 1 ? 2 : 3, OPITCH = 2 * D + 16;
  constexpr int OROWS = OP * D * OPITCH <= SH::bytes ? D : 32;  // output channels of a pass
  static_assert(OP * OROWS * OPITCH <= SH::bytes, "space of the gauge");
  const size_t gb = ((size_t(l) * 2 + 1) * G.H + h) * G.R * size_t(G.g) * G.g;
  const bool mine = 32 * w + n < rows;
  const size_t orow = (size_t(lv) * a.nsplit + sp) * a.N + (qt.tok0 + qt.i0 + tok);
  const size_t phead = orow * a.Hq + h * a.grp + j0 + jj;  // this lane's partial row
  const size_t ooff = size_t(lv) * a.o.sl + size_t(h * a.grp + j0 + jj) * a.o.sh + size_t(qt.tok0 + qt.i0 + tok) * a.o.st;
  if (a.nsplit > 1 && mine && hc == 0) {
    a.ml[2 * phead] = m == -INFINITY ? -INFINITY : m * cs;
    a.ml[2 * phead + 1] = lall;
  }
  bf16x8_t x[OP][KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    u32x4_t t[OP];
#pragma unroll
    for (int e2 = 0; e2 < 4; ++e2) {
      uint32_t o[OP];
      float x0 = O[kk >> 1][8 * (kk & 1) + 2 * e2] * inv, x1 = O[kk >> 1][8 * (kk & 1) + 2 * e2 + 1] * inv;
      if constexpr (PASS) {
        x0 = __builtin_amdgcn_ldexpf(x0, -up[1]);
        x1 = __builtin_amdgcn_ldexpf(x1, -up[1]);
      }
      split_b<OP>(x0, x1, o);
#pragma unroll
      for (int p = 0; p < OP; ++p) t[p][e2] = o[p];
    }
#pragma unroll
    for (int p = 0; p < OP; ++p) x[p][kk] = as_bf16x8(t[p]);
  }
#pragma unroll 1
  for (int ct = 0; 32 * ct < d; ++ct) {  // output channels 32 ct ..
    if (OROWS == 32 || ct == 0) {
      __syncthreads();
      stage_gauge<OP, OROWS, KK, NT>(sm, G.tr, gb, G.g, d, 32 * ct, 0);
      __syncthreads();
    }
    if (idle) continue;
    f32x16_t y = f32x16_t{};
    int c0, c1;
    reached(G.g, 32 * ct, 32, c0, c1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (16 * kk >= d || 16 * kk > c1 || 16 * kk + 15 < c0) continue;
#pragma unroll
      for (int p = 0; p < OP; ++p) {
        // element e of the sums' operand is channel 16 kk + 8 (e & 1) + 4 (e >> 2) + 2 hc + ((e & 3) >> 1)
        const uint32_t* src = reinterpret_cast<const uint32_t*>(sm + (OROWS * p + (OROWS == 32 ? 0 : 32 * ct) + n) * OPITCH + 32 * kk) + hc;
        const uint32_t c0 = src[0], c4 = src[2], c8 = src[4], c12 = src[6];
        const bf16x8_t A = as_bf16x8(u32x4_t{__builtin_amdgcn_perm(c8, c0, 0x05040100u), __builtin_amdgcn_perm(c8, c0, 0x07060302u),
                                             __builtin_amdgcn_perm(c12, c4, 0x05040100u), __builtin_amdgcn_perm(c12, c4, 0x07060302u)});
#pragma unroll
        for (int s = 0; s < OP; ++s)
          if (p + s < OP) y = mfma(A, x[s][kk], y);
      }
    }
    // lane (n, hc): channels 32 ct + 8 i + 4 hc + j of its query
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ch = 32 * ct + 8 * i + 4 * hc;
      if (!mine || ch >= d) continue;
      const float4 o = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
      if (a.nsplit > 1) {
        *reinterpret_cast<float4*>(a.part + phead * d + ch) = o;
      } else if (a.o.bf16) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.ptr) + ooff + ch) =
            make_uint2(pk_b(o.x, o.y), pk_b(o.z, o.w));
      } else {
        *reinterpret_cast<float4*>(static_cast<float*>(a.o.ptr) + ooff + ch) = o;
      }
    }
  }
}

template <int D, int PL, int BITS>
hipError_t run_chunk(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  const void* fn = reinterpret_cast<const void*>(chunk_attend<D, PL, BITS>);
  const int smem = ChunkShape<D, PL>::all;
  if (smem > 65536) {
    const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  ChunkDev av = a;
  GaugeDev gv = G;
  CodecDev cv = c;
  void* args[] = {&av, &gv, &cv};
  return hipLaunchKernel(fn, dim3(blocks), dim3(64 * NW), args, smem, st);
}

// EACH: a kernel for each code width (else one that reads it at run time)
template <int D, int PL, bool EACH>
hipError_t by_layout(const ChunkDev& a, const GaugeDev& G, const CodecDev& c, int blocks, hipStream_t st) {
  if (c.backend == CG_BACKEND_PASSTHROUGH) return run_chunk<D, PL, kErrorFree>(a, G, c, blocks, st);
  if (!chunk_wide(c, a.q.d)) return run_chunk<D, PL, kAnyLayout>(a, G, c, blocks, st);
  if constexpr (EACH) {
    switch (c.bits) {
      case 2: return run_chunk<D, PL, 2>(a, G, c, blocks, st);
      case 3: return run_chunk<D, PL, 3>(a, G, c, blocks, st);
      case 4: return run_chunk<D, PL, 4>(a, G, c, blocks, st);
      case 6: return run_chunk<D, PL, 6>(a, G, c, blocks, st);
      default: return run_chunk<D, PL, 8>(a, G, c, blocks, st);
    }
  } else {
    return run_chunk<D, PL, 0>(a, G, c, blocks, st);
  }
}

}  // namespace

}  // namespace cg
