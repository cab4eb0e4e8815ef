// Attention of trees over block-uniform pools, bf16 results: the kernel over the positions.
//
// As in the chunk attention the gauge stays outside: scores are q' . zhat^K with q' = G_K q (cg_tree_join.hip makes the
// operands), o = G_V^T sum_t p_t zhat^V_t (there, where the parts are joined).  A tree has few query rows and many positions,
// so the work is cut along the positions of all tiles in one line, in equal pieces whatever the rows' lengths, a workgroup
// each; what a workgroup finds of a tile is a part, joined later in a fixed order.
//
// A wave takes 32 positions at a time and all 32 QT query rows of the tile; no wave waits for another within a tile.
//   S^T = K Q'^T on v_mfma_f32_32x32x16_f16: lane (position n, half) holds the codes of half of a position's channels and
//     decodes them straight into its A operands (the contraction's order is free: q' is laid out to match); the query operands
//     lie in LDS, shared by the four waves
//   softmax in the lane and its partner 32 lanes away (lane: one query, half of the positions)
//   O^T += V^T P^T: values go through the wave's own LDS rows, read back transposed
// Operands are binary16 as in the chunk attention (11 bits, cg_chunk_kernel.h), and a unit with zhat beyond it, an infinity or a NaN is
// summed position by position in binary32, in a loop of its own behind the others (within theirs its registers spill).
//
// Bound by what a unit has to do in order, at two waves per SIMD.  A unit (32 positions, 64 query rows, 128 channels) is
// about 430 vector instructions and 32 products, 1720 + 1050 cycles of its SIMD, and takes 4060 of them (8 long rows; 4980
// where 32 shorter rows open and join more tiles): vector instructions issue in 46 (37)% of the cycles, products run in 28 (20)%.  A
// wave has an instruction issued in 45 (40)% of its time, waits for its turn in 24 (19)%, and for results of LDS and of
// products in 31 (40)%.  32 trees of 8 to 16 nodes behind up to 8192 positions, 8 KV heads x 4, 4 bits: 84 to 87 us over the positions
// where the bytes take 30 and the products 28; a call 105, by the chunk attention's kernel with masks 237.  Codes become
// binary16 by one conversion from 8-bit floating point for two (with a mask and a fused multiply-add 11 cycles of issue a
// pair); 3 bits, four of them to a word after six byte permutations a run: 103 us where code by code it was 124 (24 trees
// of 25 nodes behind 4096 positions, 16 KV heads x 2).  Without any load of codes a call takes 7 us less, so nothing is fetched further
// ahead; one wave per SIMD with all 512 registers, or the next unit's scores beside this one's values, took longer;
// leaving out the second group of queries in tiles of at most 32 rows won 2%, at twice the code.  Workgroups that take
// turns in priority: 1 to 2%.  A tile of 64 rows where a row's queries fill more than 32: two waves per SIMD instead of
// three, and a code is decoded half as often (a call for 8 nodes a tree takes 75 us, in tiles of 32, for 16 106).
#pragma once

#include "cg_chunk_kernel.h"
#include "cg_tree_attend.h"

namespace cg {

namespace {

template <int D, int QT, int BITS>
struct TreeShape {
  static constexpr int KS = D / 16, CT = D / 32;
  static constexpr int RB = D * BITS / 8;                 // bytes of a code row
  static constexpr int VP = 2 * D + 64;                   // V rows in binary16: 4 of them cover all banks once
  static constexpr int queries = QT * KS * 64 * 16;       // operands of the tile's queries
  static constexpr int values = 16 * VP;                  // a wave's rows
  static constexpr int codes = (32 * RB + 1023) / 1024 * 1024, sides = 32 * (D / 32) * 4;  // a wave's next keys, and values
  static constexpr int wave = values + 2 * (codes + sides);
  static constexpr int joined = 2 * QT * CT * 4096;       // two waves' sums on their way to the others
  static constexpr int all = (queries + 4 * wave > joined ? queries + 4 * wave : joined) + 4 * 32 * QT * 8;
  static_assert(wave >= 4 * 2 * D * 4, "space of the rows in binary32");
};

constexpr float kMostWeight = 16384.0f;  // 2^(kPBias + kLag)
static_assert(kPBias + kLag == 14.0f, "largest weight");

template <int D, int QT, int BITS>
__global__ __launch_bounds__(256, QT == 1 ? 3 : 2) void tree_attend(TreeRun p) {
  using SH = TreeShape<D, QT, BITS>;
  constexpr int KS = SH::KS, CT = SH::CT, VP = SH::VP, RH = D / 64, ROWS = 32 * QT, RB = SH::RB;  // RH: runs of 32 channels of a lane
  extern __shared__ __attribute__((aligned(64))) uint8_t sm[];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hc = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)sm));
  uint8_t* const mine = sm + SH::queries + w * SH::wave;  // this wave's: rows of values, codes and sides of keys, of values
  uint8_t* const vbuf = mine;
  uint8_t* const kraw = mine + SH::values;
  uint8_t* const vraw = kraw + SH::codes + SH::sides;
  float2(*ex)[ROWS] = reinterpret_cast<float2(*)[ROWS]>(sm + SH::all - 4 * ROWS * 8);
  const int inner = p.H * p.nqc, P = p.page_size;
  int bid = blockIdx.x;
  const int hq = bid % inner;
  bid /= inner;
  const int wg = bid % p.nwg, lv = bid / p.nwg;
  const int h = hq / p.nqc, qc = hq - h * p.nqc, l = lv + p.l0;
  const size_t lh = size_t(lv) * inner + hq;
  const int64_t per = p.line->per, total = p.line->total;
  int64_t at = per * wg;
  const int64_t stop = min(total, at + per);
  if (at >= stop) return;
  const int nh = min(p.heads, p.grp - qc * p.heads);
  const int nblk = D / p.n;
  const size_t prows = size_t(p.H) * P, row0 = (size_t(l) * p.pages_all * p.H + h) * P;

  for (int t = p.first[wg]; at < stop; ++t) {
    const TreeTile tile = p.tiles[t];
    const int from = int(at - tile.start), to = int(min(stop - tile.start, int64_t(tile.len)));
    at = tile.start + tile.len;
    // blocks: those that hold sinks before the window, then from the window's first position on
    const int base = tile.base, held = tile.held;
    int lo_t = 0, sink_t = 0;
    if (p.window > 0) {
      lo_t = max(0, base - p.window + 1) / kTreeBlock;
      sink_t = min((min(p.sinks, held) + kTreeBlock - 1) / kTreeBlock, lo_t);
    }
    const int v1 = to - kTileCost;
    int v = max(0, from - kTileCost);
    auto first_pos = [&](int u) { return kTreeBlock * (u < sink_t ? u : lo_t + u - sink_t) + 32 * w; };

    // ---- units: pages are looked up one ahead of the loads, which go to LDS: the next keys once these are decoded, the
    // next values once these are (always as many, so that their arrival can be counted; what is not there is not used)
    typedef const __attribute__((address_space(4))) int* scalar_ints;
    const scalar_ints table = (scalar_ints)(p.pages + size_t(tile.b) * p.max_pages);
    size_t srow = row0;   // first cache row of the unit that is fetched
    bool have = false;    // it has a page inside the pool
    int look_v = v, look_p = first_pos(v) / P, look_off = first_pos(v) - look_p * P, page = -1, off = 0;
    auto look = [&]() {
      page = look_v < v1 && look_p < p.max_pages ? table[look_p] : -1;
      off = look_off;
      look_off += kTreeBlock;
      if (++look_v == sink_t) {  // from the sinks to the window
        look_p = first_pos(look_v) / P;
        look_off = first_pos(look_v) - look_p * P;
      }
      while (look_off >= P) {
        look_off -= P;
        ++look_p;
      }
    };
    auto find = [&](int u) {
      const bool live = u < v1 && first_pos(u) < held;
      const int pg = page, o = off;
      look();
      have = pg >= 0 && pg < p.pages_all;
      if (live && !have && lane == 0 && p.err) atomicOr(p.err, CG_FLAG_POS_RANGE);
      have = have && live;
      srow = row0 + (have ? size_t(pg) * prows + o : 0);
    };
    constexpr int NL = SH::codes / 1024;  // loads of 16 bytes a lane for the codes of 32 positions
    // (written out, not by the builtin: the compiler lets every later read of LDS wait for all of them)
    auto fetch = [&](const uint8_t* codes, const uint32_t* side, const uint8_t* dst) {
      const uint8_t* src = codes + srow * RB;
      const uint32_t* sid = side + srow * nblk;
      const uint32_t to = uint32_t(dst - sm) + lds0;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const uint32_t g = 16 * min(64 * i + lane, 2 * RB - 1);  // granule (past the last one that one again)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(g), "s"(src), "s"(to + 1024 * i) : "memory");
      }
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint32_t s = 4 * min(64 * i + lane, 32 * nblk - 1);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(s), "s"(sid), "s"(to + SH::codes + 256 * i) : "memory");
      }
    };
    constexpr int NF = NL + D / 64;       // loads of a fetch
    auto landed = []() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NF) : "memory"); };  // all but the last fetch's
    auto fetch_keys = [&]() { fetch(p.kcodes, p.kside, kraw); };
    auto fetch_values = [&]() { fetch(p.vcodes, p.vside, vraw); };
    // run `run` (32 channels) of position pos, and its side word
    auto raw_run = [&](const uint8_t* src, int pos, int run) {
      Raw32 o;
      const uint32_t* x = reinterpret_cast<const uint32_t*>(src + pos * RB + run * (4 * BITS));
      if constexpr (BITS % 4 == 0) {
#pragma unroll
        for (int i = 0; i < BITS / 4; ++i) {
          const u32x4_t y = reinterpret_cast<const u32x4_t*>(x)[i];
#pragma unroll
          for (int e = 0; e < 4; ++e) o.w[4 * i + e] = y[e];
        }
      } else {
#pragma unroll
        for (int i = 0; i < BITS; ++i) o.w[i] = x[i];
      }
      if constexpr (BITS == 3) {
        // codes c, c + 8, c + 16, c + 24 lie 24 bits apart: bytes i, i + 3, i + 6, i + 9 in a word hold them at one place
        const uint32_t a = o.w[0], b = o.w[1], c = o.w[2];
        o.w[0] = __builtin_amdgcn_perm(c, __builtin_amdgcn_perm(b, a, 0x0c060300u), 0x05020100u);
        o.w[1] = __builtin_amdgcn_perm(c, __builtin_amdgcn_perm(b, a, 0x0c070401u), 0x06020100u);
        o.w[2] = __builtin_amdgcn_perm(c, __builtin_amdgcn_perm(b, a, 0x0c0c0502u), 0x07040100u);
      }
      o.side = *reinterpret_cast<const uint32_t*>(src + SH::codes + 4 * (pos * nblk + 32 * run / p.n));
      return o;
    };

    // ---- the first codes and the tile's queries
    look();
    __syncthreads();  // the queries before are read, and so is what the waves joined in
    find(v);
    fetch_keys();
    fetch_values();
    {
      const uint4* src = p.qf + (lh * p.ntile + t) * (SH::queries / 16);
#pragma unroll
      for (int i = 0; i < SH::queries / 16 / 256; ++i) reinterpret_cast<uint4*>(sm)[i * 256 + tid] = src[i * 256 + tid];
    }
    const int rows = tile.ntok * nh;
    auto token = [&](int q) { return tile.tok0 + min(32 * q + n, rows - 1) / nh; };
    float cs[QT];
    int most = base;  // the largest position of a query
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      cs[q] = p.qs[(lh * p.ntile + t) * ROWS + min(32 * q + n, rows - 1)];
      if (p.window > 0) most = max(most, p.pos[token(q)]);
    }
    if (p.window > 0) most = wave_most(most);
    // bit i: the lane's query sees position t + i (read anew: few units have hidden positions)
    auto seen_from = [&](int q, int t) {
      asm volatile("" : "+v"(t));  // (not before it is asked for)
      const int tok = token(q), plow = p.window > 0 ? max(max(p.pos[tok], base) - p.window, -1) : -1;
      return tree_seen(p.mask + size_t(tok) * p.words, p.words, base, held, plow, p.sinks, t);
    };
    const int v0 = v;
    const uint4* const qf = reinterpret_cast<const uint4*>(sm) + lane;
    __syncthreads();

    f32x16_t O[QT][CT];
    float m[QT], lsum[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      m[q] = -INFINITY;
      lsum[q] = 0.0f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) O[q][ct] = f32x16_t{};
    }
    uint32_t one = 0x64006400u, cm = ((1u << BITS) - 1u) * (BITS <= 4 ? 0x01010101u : 0x00010001u);
    asm("" : "+v"(one), "+v"(cm));
    // side word of a run as the pairs' operands; true if its zhat are not all in binary16 (its largest code's is not)
    auto ranges = [&](uint32_t s, f16x2_t& mn, f16x2_t& sc) {
      const _Float16 m1 = __builtin_bit_cast(_Float16, uint16_t(s)), s1 = __builtin_bit_cast(_Float16, uint16_t(s >> 16));
      mn = f16x2_t{m1, m1};
      sc = f16x2_t{s1, s1};
      return !__builtin_isfinite(__builtin_fmaf16(s1, (_Float16)((1 << BITS) - 1), m1));
    };
    // granule g of a run: 8 channels as pairs (tree_channel)
    auto granule = [&](const Raw32& rw, int g, f16x2_t mn, f16x2_t sc) {
      u32x4_t o;
      if constexpr (BITS == 3) {
        const uint32_t* z = rw.w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = 2 * g + (j >> 1);  // of 8: at bit 3 c of the words' bytes in a row
          const uint32_t by = c == 2   ? ((z[0] >> 6) & 0x03030303u) | ((z[1] << 2) & 0x04040404u)
                              : c == 5 ? ((z[1] >> 7) & 0x01010101u) | ((z[2] << 1) & 0x06060606u)
                              : c == 3 ? z[1] & (cm << 1)  // twice the codes
                                       : (z[3 * c / 8] >> (3 * c % 8)) & cm;
          const float of = c == 3 ? 256.0f : 512.0f;
          const f16x2_t q = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(by, of, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(by, of, false);
          o[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(q, sc, mn));
        }
      } else if constexpr (BITS == 4 || BITS == 2) {
        // a code alone in a byte is 2^-9 of it in 8-bit floating point (e4m3: numbers below 2^-5 are multiples of
        // 2^-9), so one conversion makes binary16 of two
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t by = BITS == 4 ? (rw.w[g] >> (4 * (j >> 1))) & cm : (rw.w[g >> 1] >> (2 * j)) & cm;
          const f16x2_t q = (BITS == 4 ? j & 1 : g & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(by, 512.0f, true)
                                                        : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(by, 512.0f, false);
          o[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(q, sc, mn));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(int_pair(code_pair(rw.w, BITS, g >> 1, g & 1, j, one, cm)), sc, mn));
      }
      return o;
    };
    // values: lane (position, quarter of the channels) writes; element e of an operand is position 8 (e / 4) + 4 hc + e % 4
    const int vpos = lane >> 2, vrun = (lane & 3) * RH / 2;
    const uint32_t vdst = uint32_t(vbuf - sm) + vpos * VP + (lane & 3) * (D / 2) + 16 * (vpos & 3);
    const uint8_t* const vb = vbuf + (4 * hc + ((lane >> 2) & 3)) * VP +
                              16 * ((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ ((lane >> 2) & 3)) + 8 * (lane & 1);
    auto vfrag = [&](int ct) {
      typedef __attribute__((address_space(3))) s16x4_t* lds4;
      const s16x4_t y0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vb + 64 * ct));
      const s16x4_t y1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vb + 64 * ct + 8 * VP));
      return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Workgroups on a CU would go by age, the last to finish alone: they take turns in going first
    constexpr int TURNS = QT == 1 ? 3 : 2;
    int prio = int(blockIdx.x / ((gridDim.x + TURNS - 1) / TURNS));
    bool left = false;  // units that binary16 does not hold
    for (; v < v1; ++v) {
      const int t0 = first_pos(v);
      if (t0 >= held) break;
      if (++prio >= TURNS) prio = 0;
      if (prio == 0) __builtin_amdgcn_s_setprio(0);
      else if (prio == 1) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(2);
      const bool none = !have;  // nothing of a page outside the pool; positions from `held` on are zeros (their bytes may hold anything)
      const int live = none ? 0 : held - t0;
      landed();
      Raw32 rk[RH];
#pragma unroll
      for (int r = 0; r < RH; ++r) rk[r] = raw_run(kraw, n, hc * RH + r);
      bool st = false;
      f16x2_t kmn[RH], ksc[RH];
#pragma unroll
      for (int r = 0; r < RH; ++r) {
        if (live < 32 && n >= live) rk[r].side = 0u;
        st |= ranges(rk[r].side, kmn[r], ksc[r]);
      }
      // scores; operands a step ahead
      f32x16_t S[QT];
#pragma unroll
      for (int q = 0; q < QT; ++q) S[q] = f32x16_t{};
      u32x4_t kf[2];
      uint4 qx[2][QT];
#pragma unroll
      for (int q = 0; q < QT; ++q) qx[0][q] = qf[q * KS * 64];
      kf[0] = granule(rk[0], 0, kmn[0], ksc[0]);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        if (k + 1 < KS) {
#pragma unroll
          for (int q = 0; q < QT; ++q) qx[(k + 1) & 1][q] = qf[(q * KS + k + 1) * 64];
          kf[(k + 1) & 1] = granule(rk[(k + 1) >> 2], (k + 1) & 3, kmn[(k + 1) >> 2], ksc[(k + 1) >> 2]);
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) S[q] = mfma_h(as_f16x8(kf[k & 1]), __builtin_bit_cast(f16x8_t, qx[k & 1][q]), S[q]);
        __builtin_amdgcn_sched_group_barrier(0x100, QT, 0);
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 16 / QT, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      find(v + 1);
      fetch_keys();
      // the values' ranges: both halves of the unit, before any weight is formed
      uint32_t vside[2];
      landed();
#pragma unroll
      for (int kp = 0; kp < 2; ++kp) {
        const int pos = 16 * kp + vpos;
        vside[kp] = *reinterpret_cast<const uint32_t*>(vraw + SH::codes + 4 * (pos * nblk + 32 * vrun / p.n));
        if (live < 32 && pos >= live) vside[kp] = 0u;
        f16x2_t mn, sc;
        st |= ranges(vside[kp], mn, sc);
      }
      const bool odd = __builtin_amdgcn_ballot_w64(st) != 0;
      if (odd) {  // summed after the others: nothing of it here
        left = true;
        vside[0] = vside[1] = 0u;
      }
      // hidden positions
      const bool whole = !odd && !none && t0 + 32 <= base && (p.window == 0 || t0 > most - p.window || t0 + 32 <= p.sinks);
      f16x8_t W[QT][2];  // weights
      auto weigh = [&](int q) {
        const float o = kPBias - (m[q] == -INFINITY ? 0.0f : m[q] * cs[q]);
        float ls[2] = {0.0f, 0.0f};
#pragma unroll
        for (int kp = 0; kp < 2; ++kp) {
          u32x4_t f;
#pragma unroll
          for (int e2 = 0; e2 < 4; ++e2) {
            const int e = 8 * kp + 2 * e2;
            f[e2] = pk_h(__builtin_amdgcn_exp2f(fmaf(S[q][e], cs[q], o)), __builtin_amdgcn_exp2f(fmaf(S[q][e + 1], cs[q], o)));
            // the rounded weights, as the values meet them (v_dot2_f32_f16 adds both to binary32 exactly)
            const f16x2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
            ls[e2 & 1] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, uint32_t(f[e2])), ones, ls[e2 & 1], false);
          }
          W[q][kp] = as_f16x8(f);
        }
        return ls[0] + ls[1];
      };
      // Weights relative to the largest score so far, before this unit's scores are compared with it: while their sum is at most
      // 2^(kPBias + kLag) none of them passes what binary16 holds, and the largest score may stay what it was.  Seldom not:
      // then it is found, and they are formed again (8 trees of 60 nodes 196 -> 190 us a call)
      float ls[QT];
      bool again = false;
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        if (!whole) {
          const uint32_t seen = odd || none ? 0u : uint32_t(seen_from(q, t0 + 4 * hc));
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t keep = uint32_t(__builtin_amdgcn_sbfe(int(seen), 8 * (e >> 2) + (e & 3), 1));
            S[q][e] = __uint_as_float((__float_as_uint(S[q][e]) & keep) | (0xff800000u & ~keep));
          }
        }
        ls[q] = weigh(q);
        again |= m[q] == -INFINITY || !(ls[q] <= kMostWeight);
      }
      if (__builtin_amdgcn_ballot_w64(again)) {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          float mx = S[q][0];
#pragma unroll
          for (int e = 1; e < 16; ++e) mx = fmaxf(mx, S[q][e]);
          mx = halves_max(mx);
          const float mn = fmaxf(m[q], mx);
          const float al = mn == m[q] ? 1.0f : __builtin_amdgcn_exp2f((m[q] - mn) * cs[q]);
          m[q] = mn;
          lsum[q] *= al;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) O[q][ct][e] *= al;
          ls[q] = weigh(q);
        }
      }
#pragma unroll
      for (int q = 0; q < QT; ++q) lsum[q] += ls[q];
      // values, 16 positions at a time through the wave's rows
#pragma unroll
      for (int kp = 0; kp < 2; ++kp) {
        const int pos = 16 * kp + vpos;
        f16x2_t mn, sc;
        ranges(vside[kp], mn, sc);
        if constexpr (D == 128) {
          const Raw32 rv = raw_run(vraw, pos, vrun);
#pragma unroll
          for (int g = 0; g < 4; ++g) *reinterpret_cast<u32x4_t*>(sm + (vdst ^ (16 * g))) = granule(rv, g, mn, sc);
        } else {
          // half a run
          const Raw32 rv = raw_run(vraw, pos, vrun);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const u32x4_t lo = granule(rv, g, mn, sc), hi = granule(rv, g + 2, mn, sc);
            const int odd_half = lane & 1;
            u32x4_t o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = odd_half ? hi[e] : lo[e];
            *reinterpret_cast<u32x4_t*>(sm + ((uint32_t(vbuf - sm) + vpos * VP + 64 * vrun + 16 * (vpos & 3)) ^ (16 * (g + 2 * odd_half)))) = o;
          }
        }
        __builtin_amdgcn_wave_barrier();
        f16x8_t vf[2];
        vf[0] = vfrag(0);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if (ct + 1 < CT) vf[(ct + 1) & 1] = vfrag(ct + 1);
#pragma unroll
          for (int q = 0; q < QT; ++q) O[q][ct] = mfma_h(vf[ct & 1], W[q][kp], O[q][ct]);
        }
        __builtin_amdgcn_wave_barrier();  // the rows are read before the next ones are written
      }
      fetch_values();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing comes to LDS any more)

    if (left) {
      CacheDev kc{const_cast<uint8_t*>(p.kcodes), const_cast<uint32_t*>(p.kside)}, vc{const_cast<uint8_t*>(p.vcodes), const_cast<uint32_t*>(p.vside)};
      CodecDev cd{};
      cd.bits = BITS;
      cd.n = p.n;
      // those units, position by position in binary32, four at a time through the wave's space
      float* rows32 = reinterpret_cast<float*>(mine);
#pragma unroll 1
      for (v = v0; v < v1 && first_pos(v) < held; ++v) {
        const int t0 = first_pos(v), live = min(32, held - t0), pg = table[t0 / P];
        if (pg < 0 || pg >= p.pages_all) continue;
        const size_t crow = row0 + size_t(pg) * prows + t0 % P;
        bool st = false;
#pragma unroll 1
        for (int x = lane; x < 64 * nblk; x += 64) {
          f16x2_t mn, sc;
          const int y = x >> 1;  // (position, block) of the keys, of the values
          const uint32_t* side = (x & 1) ? p.vside : p.kside;
          if (y / nblk < live) st |= ranges(side[crow * nblk + y], mn, sc);
        }
        if (!__builtin_amdgcn_ballot_w64(st)) continue;
#pragma unroll 1
        for (int s0 = 0; s0 < live; s0 += 4) {
          __builtin_amdgcn_wave_barrier();
#pragma unroll 1
          for (int x = lane; x < 2 * 4 * (D / 4); x += 64) {
            const bool val = x >= 4 * (D / 4);
            const int y = val ? x - 4 * (D / 4) : x, pos = y / (D / 4), ch = 4 * (y % (D / 4));
            float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (s0 + pos < live) load4<false>(val ? vc : kc, cd, crow + s0 + pos, D, ch, z);
            *reinterpret_cast<float4*>(rows32 + (val ? 4 * D : 0) + pos * D + ch) = make_float4(z[0], z[1], z[2], z[3]);
          }
          __builtin_amdgcn_wave_barrier();
#pragma unroll 1
          for (int u = 0; u < min(4, live - s0); ++u) {
            const float *kr = rows32 + u * D + hc * (D / 2), *vr = rows32 + (4 + u) * D;
#pragma unroll
            for (int q = 0; q < QT; ++q) {
              const bool seen = (seen_from(q, t0 + s0 + u) & 1) != 0;
              float s = 0.0f;
#pragma unroll 1
              for (int k = 0; k < KS; ++k) {
                const uint4 f = qf[(q * KS + k) * 64];
                const float* kc = kr + 32 * (k >> 2);
                const uint32_t fw[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  s = fmaf(h_hi(fw[j]), kc[tree_channel(BITS, k & 3, j, 1)], fmaf(h_lo(fw[j]), kc[tree_channel(BITS, k & 3, j, 0)], s));
              }
              s = halves_sum(s);
              const float mn = seen ? fmaxf(m[q], s) : m[q];
              const float al = m[q] == mn ? 1.0f : __builtin_amdgcn_exp2f((m[q] - mn) * cs[q]);
              const float pr = seen ? __builtin_amdgcn_exp2f(fmaf(s, cs[q], kPBias - (mn == -INFINITY ? 0.0f : mn * cs[q]))) : 0.0f;
              m[q] = mn;
              lsum[q] = fmaf(lsum[q], al, hc ? 0.0f : pr);
#pragma unroll
              for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float o = O[q][ct][e] * al;
                  const int ch = 32 * ct + tree_channel(BITS, e >> 2, 2 * hc + ((e & 3) >> 1), e & 1);
                  O[q][ct][e] = seen ? fmaf(pr, vr[ch], o) : o;
                }
            }
          }
        }
      }
    }

    // ---- the four waves' sums, joined: everything relative to the largest maximum, then waves 2 and 3 to 0 and 1, and what
    // these hold by all four
    float M[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      lsum[q] = halves_sum(lsum[q]);
      if (hc == 0) ex[w][32 * q + n] = make_float2(m[q], lsum[q]);
    }
    __syncthreads();  // (every wave is through with its rows)
    const size_t slot = lh * (p.nwg + p.ntile) + wg + t;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      float2 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = ex[i][32 * q + n];
      M[q] = fmaxf(fmaxf(y[0].x, y[1].x), fmaxf(y[2].x, y[3].x));
      auto scale = [&](float v) { return v == M[q] ? 1.0f : __builtin_amdgcn_exp2f((v - M[q]) * cs[q]); };
      const float al = scale(m[q]);
      if (w == 0 && hc == 0)
        p.ml[slot * ROWS + 32 * q + n] = make_float2(M[q] == -INFINITY ? -INFINITY : M[q] * cs[q],
                                                     y[0].y * scale(y[0].x) + y[1].y * scale(y[1].x) + y[2].y * scale(y[2].x) + y[3].y * scale(y[3].x));
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[q][ct][e] = al == 0.0f ? 0.0f : O[q][ct][e] * al;
    }
    // (all of LDS but the exchanged maxima; the queries are read)
    float4* const jb = reinterpret_cast<float4*>(sm);  // [2][QT][CT][4][64]
    auto put = [&](int side) {
#pragma unroll
      for (int q = 0; q < QT; ++q)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int f = 0; f < 4; ++f)
            jb[(((side * QT + q) * CT + ct) * 4 + f) * 64 + lane] =
                make_float4(O[q][ct][4 * f], O[q][ct][4 * f + 1], O[q][ct][4 * f + 2], O[q][ct][4 * f + 3]);
    };
    if (w >= 2) put(w - 2);
    __syncthreads();
    if (w < 2) {
#pragma unroll
      for (int q = 0; q < QT; ++q)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            const float4 y = jb[(((w * QT + q) * CT + ct) * 4 + f) * 64 + lane];
            O[q][ct][4 * f] += y.x;
            O[q][ct][4 * f + 1] += y.y;
            O[q][ct][4 * f + 2] += y.z;
            O[q][ct][4 * f + 3] += y.w;
          }
      put(w);  // (where the wave has just read)
    }
    __syncthreads();
    float4* const dst = reinterpret_cast<float4*>(p.part) + slot * (QT * CT * 4 * 64) + lane;
#pragma unroll
    for (int i = 0; i < QT * CT; ++i) {  // a quarter of every channel tile's sums each
      const int at = 4 * i + w;
      const float4 x = jb[at * 64 + lane], y = jb[(QT * CT * 4 + at) * 64 + lane];
      dst[at * 64] = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
    }
  }
}

template <int D, int QT, int BITS>
hipError_t run_tree_attend(const TreeRun& p, int blocks, hipStream_t st) {
  const void* fn = reinterpret_cast<const void*>(tree_attend<D, QT, BITS>);
  const int smem = TreeShape<D, QT, BITS>::all;
  if (smem > 65536) {
    const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  TreeRun pv = p;
  void* args[] = {&pv};
  return hipLaunchKernel(fn, dim3(blocks), dim3(256), args, smem, st);
}

template <int D, int QT>
hipError_t tree_by_bits(const TreeRun& p, int bits, int blocks, hipStream_t st) {
  switch (bits) {
    case 2: return run_tree_attend<D, QT, 2>(p, blocks, st);
    case 3: return run_tree_attend<D, QT, 3>(p, blocks, st);
    case 4: return run_tree_attend<D, QT, 4>(p, blocks, st);
    case 6: return run_tree_attend<D, QT, 6>(p, blocks, st);
    default: return run_tree_attend<D, QT, 8>(p, blocks, st);
  }
}

}  // namespace

}  // namespace cg
