// Attention of trees: the tiles and the line of their blocks, the queries' operands, and the joining of the parts.
#include <algorithm>

#include "cg_chunk_kernel.h"
#include "cg_tree_attend.h"

namespace cg {

namespace {

// The plan (workgroup 0, beside those that make the queries' operands: nothing there waits for it): every row's tiles, in
// order, on one line of blocks, cut into `nwg` equal pieces, but of at least kLeast blocks and half the root of the longest
// tile's (a few long rows: a piece costs about 1.3 us a block, joining about 0.4 us a part).  32 short trees behind 200
// positions: pieces of at least 1, 2, 4, 8 blocks 43, 43, 42, 50 us a call; one tree behind 30000: 4, 8, 12 blocks 68, 58, 61.  A thread takes a
// row at a time.
constexpr int kPlanThreads = 512;
constexpr int kLeast = 4;

__device__ __forceinline__ int tree_blocks(const ChunkDev& a, int base, int held) {
  if (held <= 0) return kTileCost;
  int lo_t = 0, sink_t = 0;
  if (a.window > 0) {
    lo_t = max(0, base - a.window + 1) / kTreeBlock;
    sink_t = min((min(a.sinks, held) + kTreeBlock - 1) / kTreeBlock, lo_t);
  }
  return kTileCost + sink_t + (held - 1) / kTreeBlock - lo_t + 1;
}

__device__ void tree_line(const TreeDev& p) {
  const ChunkDev& a = p.c;
  __shared__ int64_t sums[2][kPlanThreads / 64];
  __shared__ int longest;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int turn = 0, most = 0;
  if (tid == 0) longest = 0;
  // sum of v over the threads before this one, and over all
  auto scan = [&](int64_t v, int64_t& all) {
    int64_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(s, o);
      if (lane >= o) s += y;
    }
    if (lane == 63) sums[turn][w] = s;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int i = 0; i < kPlanThreads / 64; ++i) {
      if (i < w) s += sums[turn][i];
      all += sums[turn][i];
    }
    turn ^= 1;
    return s - v;
  };
  // this thread's row of a round: its tiles (none past the room there is: rows that overlap may ask for more), the
  // first one's number and place
  int c0, n, held, base, nt, len;
  int64_t first, at, tiles, total;
  auto round = [&](int b0, int64_t tiles0, int64_t total0, bool flag) {
    const int b = b0 + tid;
    c0 = n = held = base = nt = len = 0;
    if (b < a.B) {
      held = a.lens[b];
      n = row_tokens(a, b, c0);
      bool bad = n < 0;
      if (n > 0) {
        if (held < n || held > a.cap) {
          bad = true;
          held = 0;
        }
        base = held ? held - n : 0;
        nt = (n + a.tq - 1) / a.tq;
        len = tree_blocks(a, base, held);
      }
      if (flag && bad && a.err) atomicOr(a.err, CG_FLAG_POS_RANGE);
    }
    first = tiles0 + scan(nt, tiles);
    nt = int(max(int64_t(0), min(int64_t(nt), a.ntile - first)));
    at = total0 + scan(int64_t(nt) * len, total);
    tiles += tiles0;
    total += total0;
  };
  // the line's length first; one round holds most batches' rows
  int64_t tiles0 = 0, total0 = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    round(b0, tiles0, total0, true);
    most = max(most, len);
    tiles0 = tiles;
    total0 = total;
  }
  if (most) atomicMax(&longest, most);
  __syncthreads();
  const int64_t least = max(kLeast, int(ceilf(0.5f * sqrtf(float(longest)))));
  const int64_t line = total0, per = max(least, (line + p.nwg - 1) / p.nwg);
  if (tid == 0) *p.line = TreeLine{line, per};
  for (int i = int(min(tiles0, int64_t(a.ntile))) + tid; i < a.ntile; i += kPlanThreads) p.tiles[i] = TreeTile{line, 0, -1, 0, 0, 0, 0, 0, -1};
  tiles0 = total0 = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    if (a.B > kPlanThreads) {
      round(b0, tiles0, total0, false);
      tiles0 = tiles;
      total0 = total;
    }
    for (int i = 0; i < nt; ++i, at += len) {
      const int t = int(first) + i;
      const int64_t g0 = at / per, g1 = (at + len - 1) / per;
      p.tiles[t] = TreeTile{at, len, b0 + tid, c0 + i * a.tq, min(a.tq, n - i * a.tq), base, held, int(g0), int(g1)};
      for (int64_t g = g0 + (g0 * per < at); g <= g1; ++g) p.first[g] = t;
    }
  }
}

// Tile `tile` of the batch, as tree_line numbers them: its row, first token and tokens
__device__ __forceinline__ bool query_tile(const ChunkDev& a, int tile, int& tok0, int& ntok) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int c0 = 0, n = 0;
    if (b0 + lane < a.B) n = row_tokens(a, b0 + lane, c0);
    const int nt = n > 0 ? (n + a.tq - 1) / a.tq : 0;
    int sum = nt;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o);
      if (lane >= o) sum += v;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(tile < before + sum);
    if (hit) {  // (the first row whose tiles pass it)
      const int src = __builtin_ctzll(hit), i0 = (tile - before - (__shfl(sum, src) - __shfl(nt, src))) * a.tq;
      tok0 = __builtin_amdgcn_readfirstlane(__shfl(c0, src) + i0);
      ntok = __builtin_amdgcn_readfirstlane(min(a.tq, __shfl(n, src) - i0));
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

// q' = G_K q of a tile's queries as the operands that tree_attend reads, one wave per 32 queries and channel tile (or more
// of them), from the bf16 matrix cores (two split planes of G as in the chunk attention; three of binary32 queries).
// Latency: 8.0 us for 256 tiles of 64 rows, with eight waves that fetch queries and gauge together (10.4 with four, the gauge
// before the tile was known).
template <int D, int QT>
__global__ __launch_bounds__(kPlanThreads) void tree_queries(TreeDev p, GaugeDev G) {
  constexpr int KK = D / 16, CT = D / 32, PARTS = kPlanThreads / 64 / QT, PER = CT >= PARTS ? CT / PARTS : 1, RH = D / 64;
  const ChunkDev& a = p.c;
  if (blockIdx.x == 0) {
    tree_line(p);
    return;
  }
  __shared__ float mxs[kPlanThreads / 64][32];
  const int lane = threadIdx.x & 63, n = lane & 31, hc = lane >> 5, w = threadIdx.x >> 6, q = w % QT, part = w / QT;
  const int inner = a.kc.H * a.nqc;
  int bid = blockIdx.x - 1;
  const int hq = bid % inner;
  bid /= inner;
  const int t = bid % a.ntile, lv = bid / a.ntile, h = hq / a.nqc, qc = hq - h * a.nqc, l = lv + a.l0;
  const size_t gb = ((size_t(l) * 2 + 0) * G.H + h) * G.R * size_t(G.g) * G.g;
  const bool on = PER * part < CT;
  int g0 = 0, g1 = -1;
  if (on) reached(G.g, 32 * PER * part, 32 * PER, g0, g1);
  // the gauge comes to LDS in whole rows (operands straight from memory are 64 pieces of 64 lines a load: 15 us a call
  // where whole rows took 9)
  constexpr int GPITCH = 2 * D + 16;
  __shared__ __attribute__((aligned(16))) uint8_t gs[2 * D * GPITCH];
  int tok0, ntok;
  if (!query_tile(a, t, tok0, ntok)) return;
  const int j0 = qc * a.heads, nh = min(a.heads, a.grp - j0), rows = ntok * nh;
  const int r = min(32 * q + n, rows - 1), tok = r / nh, jj = r - tok * nh;
  const size_t qoff = size_t(lv) * a.q.sl + size_t(h * a.grp + j0 + jj) * a.q.sh + size_t(tok0 + tok) * a.q.st;
  u32x4_t xb[KK];  // bf16 queries, on their way with the gauge
  if (on && a.q.bf16) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) xb[kk] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.q.ptr) + qoff + 16 * kk + 8 * hc);
  }
  stage_gauge<2, D, KK, kPlanThreads, 8>(gs, G.hi, gb, G.g, D, 0, 0);
  __syncthreads();
  auto operand = [&](int i, int pl, int kk) {
    return as_bf16x8(*reinterpret_cast<const u32x4_t*>(gs + (pl * D + 32 * (PER * part + i) + n) * GPITCH + 32 * kk + 16 * hc));
  };
  f32x16_t z[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) z[i] = f32x16_t{};
  float mx = 0.0f;
  if (on) {
    if (a.q.bf16) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (16 * kk > g1 || 16 * kk + 15 < g0) continue;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int pl = 0; pl < 2; ++pl) z[i] = mfma(operand(i, pl, kk), as_bf16x8(xb[kk]), z[i]);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (16 * kk > g1 || 16 * kk + 15 < g0) continue;
        const float* src = static_cast<const float*>(a.q.ptr) + qoff + 16 * kk + 8 * hc;
        u32x4_t x[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t o[3];
          split_b<3>(src[2 * e], src[2 * e + 1], o);
#pragma unroll
          for (int s = 0; s < 3; ++s) x[s][e] = o[s];
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int pl = 0; pl < 2; ++pl)
#pragma unroll
            for (int s = 0; s < 3; ++s)
              if (pl + s < 3) z[i] = mfma(operand(i, pl, kk), as_bf16x8(x[s]), z[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fabsf(z[i][e]));
  }
  mx = halves_max(mx);
  if (hc == 0) mxs[w][n] = mx;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PARTS; ++i) mx = fmaxf(mx, mxs[QT * i + q][n]);
  if (!on) return;
  const int ex = mx > 0.0f && mx < INFINITY ? __builtin_amdgcn_frexp_expf(mx) : 0;
  const float sign = a.scale < 0.0f ? -1.0f : (a.scale > 0.0f ? 1.0f : 0.0f);
  // the largest to [2^14, 2^15), as binary16's least step would otherwise take bits from the small ones
  const float cs = a.scale == 0.0f ? 1.0f : fmaxf(__builtin_amdgcn_ldexpf(fabsf(a.scale) * kLog2e, ex - 15), 1e-37f);
  const size_t lt = (size_t(lv) * inner + hq) * a.ntile + t;
  if (part == 0 && hc == 0) p.qs[lt * 32 * QT + 32 * q + n] = cs;
  // element e of channel tile ct: channel 8 (e / 4) + 4 hc + e % 4 of the tile's run
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int ct = PER * part + i;
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = sign * __builtin_amdgcn_ldexpf(z[i][e], 15 - ex);
    auto put = [&](int g, const uint32_t (&o)[4]) {
      p.qf[((lt * QT + q) * KK + 4 * (ct % RH) + g) * 64 + n + 32 * (ct / RH)] = make_uint4(o[0], o[1], o[2], o[3]);
    };
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint32_t o[4];
      if (p.bits == 4) {  // every other dword of granules 2 kk and 2 kk + 1 lies in each lane half, which write one each
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const auto u = __builtin_amdgcn_permlane32_swap(pk_h(x[8 * kk + i], x[8 * kk + i + 2]), pk_h(x[8 * kk + 4 + i], x[8 * kk + 4 + i + 2]), false, false);
          o[2 * i] = u[0];
          o[2 * i + 1] = u[1];
        }
      } else if (p.bits == 2) {  // ... part 0 and 1
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * kk + j]), __float_as_uint(x[8 * kk + 4 + j]), false, false);
          o[j] = pk_h(__uint_as_float(u[0]), __uint_as_float(u[1]));
        }
      } else if (p.bits == 3) {  // granules 2 hc and 2 hc + 1 lie in the lane
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pk_h(x[8 * (j & 1) + 2 * kk + (j >> 1)], x[8 * (j & 1) + 2 * kk + (j >> 1) + 4]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pk_h(x[8 * kk + j], x[8 * kk + 4 + j]);
      }
      put(p.bits == 3 ? 2 * hc + kk : 2 * kk + hc, o);
    }
  }
}

// The parts of a tile joined: o = G_V^T (sum_s w_s O_s / sum_s w_s l_s), w_s = 2^(m_s - max m).  A wave takes one group of
// 32 queries, one channel tile and every GR-th part; then the gauge, an output tile per wave.  11.5 us for 256 tiles of
// 64 rows in 3 parts each: 25 MB of parts beside a chain of loads (the first parts fetched with the gauge: no faster).
template <int D, int QT>
__global__ __launch_bounds__(512) void tree_join(TreeDev p, GaugeDev G) {
  constexpr int KK = D / 16, CT = D / 32, GR = 8 / (QT * CT) > 0 ? 8 / (QT * CT) : 1, PITCH = D + 4;
  static_assert(QT * CT * GR == 8, "eight waves");
  const ChunkDev& a = p.c;
  __shared__ __attribute__((aligned(16))) float o[32 * QT][PITCH];
  __shared__ __attribute__((aligned(16))) float4 sums[GR > 1 ? (GR - 1) * QT * CT * 4 * 64 : 1];
  const int lane = threadIdx.x & 63, n = lane & 31, hc = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), q = w % QT, ct = w / QT % CT, gr = w / (QT * CT);
  const int inner = a.kc.H * a.nqc;
  int bid = blockIdx.x;
  const int hq = bid % inner;
  bid /= inner;
  const int t = bid % a.ntile, lv = bid / a.ntile, h = hq / a.nqc, qc = hq - h * a.nqc, l = lv + a.l0;
  // the gauge first, in whole rows: it depends on nothing that is read here
  const size_t gb = ((size_t(l) * 2 + 1) * G.H + h) * G.R * size_t(G.g) * G.g;
  int g0, g1;
  reached(G.g, 32 * ct, 32, g0, g1);
  constexpr int GPITCH = 2 * D + 16;
  __shared__ __attribute__((aligned(16))) uint8_t gs[2 * D * GPITCH];
  stage_gauge<2, D, KK, 512, 8>(gs, G.tr, gb, G.g, D, 0, 0);
  const TreeTile tile = p.tiles[t];
  if (tile.len == 0) return;
  const int w0 = tile.wg0, w1 = tile.wg1;
  const size_t lh = size_t(lv) * inner + hq, slot0 = lh * (p.nwg + a.ntile) + t;
  const float2* ml = p.ml + slot0 * (32 * QT) + 32 * q + n;
  constexpr int UN = 4;  // parts read together
  float M = -INFINITY;
  for (int s0 = w0; s0 <= w1; s0 += UN) {
    float y[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) y[i] = ml[size_t(min(s0 + i, w1)) * (32 * QT)].x;
#pragma unroll
    for (int i = 0; i < UN; ++i) M = fmaxf(M, y[i]);
  }
  float L = 0.0f;
  f32x16_t x = f32x16_t{};
  const float4* part = reinterpret_cast<const float4*>(p.part) + slot0 * (QT * CT * 4 * 64) + (q * CT + ct) * 4 * 64 + lane;
  for (int s0 = w0 + gr; s0 <= w1; s0 += UN * GR) {
    float2 y[UN];
    float4 v[UN][4];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const size_t s = min(s0 + i * GR, w1);
      y[i] = ml[s * (32 * QT)];
#pragma unroll
      for (int f = 0; f < 4; ++f) v[i][f] = part[s * (QT * CT * 4 * 64) + f * 64];
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      if (s0 + i * GR > w1) break;
      const float ws = y[i].y == 0.0f ? 0.0f : (y[i].x == M ? 1.0f : __builtin_amdgcn_exp2f(y[i].x - M));
      L = fmaf(ws, y[i].y, L);
      if (ws != 0.0f) {  // (0 times an infinity is not 0)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          x[4 * f] = fmaf(ws, v[i][f].x, x[4 * f]);
          x[4 * f + 1] = fmaf(ws, v[i][f].y, x[4 * f + 1]);
          x[4 * f + 2] = fmaf(ws, v[i][f].z, x[4 * f + 2]);
          x[4 * f + 3] = fmaf(ws, v[i][f].w, x[4 * f + 3]);
        }
      }
    }
  }
  __shared__ float lsum[GR][QT * CT][64];
  if constexpr (GR > 1) {
    lsum[gr][q * CT + ct][lane] = L;
    if (gr) {
#pragma unroll
      for (int f = 0; f < 4; ++f)
        sums[(((gr - 1) * QT + q) * CT + ct) * 256 + f * 64 + lane] = make_float4(x[4 * f], x[4 * f + 1], x[4 * f + 2], x[4 * f + 3]);
    }
    __syncthreads();
    if (gr == 0) {
#pragma unroll
      for (int i = 1; i < GR; ++i) {
        L += lsum[i][q * CT + ct][lane];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const float4 v = sums[(((i - 1) * QT + q) * CT + ct) * 256 + f * 64 + lane];
          x[4 * f] += v.x;
          x[4 * f + 1] += v.y;
          x[4 * f + 2] += v.z;
          x[4 * f + 3] += v.w;
        }
      }
    }
  }
  if (gr == 0) {
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;  // nothing visible: zeros
#pragma unroll
    for (int e = 0; e < 16; ++e)
      o[32 * q + n][32 * ct + tree_channel(p.bits, e >> 2, 2 * hc + ((e & 3) >> 1), e & 1)] = x[e] * inv;
  }
  __syncthreads();
  if (gr) return;
  const int j0 = qc * a.heads, nh = min(a.heads, a.grp - j0), r = 32 * q + n;
  f32x16_t y = f32x16_t{};
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    if (16 * kk > g1 || 16 * kk + 15 < g0) continue;
    const int ch = 16 * kk + 8 * hc;
    const float* src = &o[r][ch];
    u32x4_t b[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t s[2];
      split_b<2>(src[2 * e], src[2 * e + 1], s);
      b[0][e] = s[0];
      b[1][e] = s[1];
    }
    const uint8_t* row = gs + (32 * ct + n) * GPITCH + 32 * kk + 16 * hc;
    const bf16x8_t A0 = as_bf16x8(*reinterpret_cast<const u32x4_t*>(row)), A1 = as_bf16x8(*reinterpret_cast<const u32x4_t*>(row + D * GPITCH));
    y = mfma(A0, as_bf16x8(b[0]), y);
    y = mfma(A0, as_bf16x8(b[1]), y);
    y = mfma(A1, as_bf16x8(b[0]), y);
  }
  if (r >= tile.ntok * nh) return;
  const int tok = r / nh, jj = r - tok * nh;
  uint16_t* out = static_cast<uint16_t*>(a.o.ptr) + size_t(lv) * a.o.sl + size_t(h * a.grp + j0 + jj) * a.o.sh + size_t(tile.tok0 + tok) * a.o.st;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint2*>(out + 32 * ct + 8 * i + 4 * hc) = make_uint2(pk_b(y[4 * i], y[4 * i + 1]), pk_b(y[4 * i + 2], y[4 * i + 3]));
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace

bool tree_attend_supported(const CodecDev& c, int d, int grp, bool bf16_out) {
  return bf16_out && c.backend == CG_BACKEND_BLOCK_UNIFORM && c.n % 32 == 0 && (d == 64 || d == 128) && grp <= 64;
}

TreePlan tree_plan(int nl, int N, int B, int max_q, int H, int Hq, int d) {
  TreePlan p;
  const int grp = Hq / H;
  const int64_t mq = std::min(max_q, N);
  p.qt = mq * grp <= 32 ? 1 : 2;
  const int M = 32 * p.qt;
  p.heads = std::min(grp, M);
  p.nqc = (grp + p.heads - 1) / p.heads;
  p.tq = M / p.heads;
  const int rows = std::min(N, B);
  p.ntile = int(std::min<int64_t>(int64_t(N) / p.tq + rows, std::min<int64_t>(N, int64_t(rows) * ((mq + p.tq - 1) / p.tq))));
  const int64_t lh = int64_t(nl) * H * p.nqc;
  // as many workgroups as LDS and registers let run at once
  p.nwg = int(std::max<int64_t>(1, (p.qt == 1 ? 3 : 2) * cu_count() / lh));
  size_t off = 256;
  p.off_tiles = off;
  off = up256(off + sizeof(TreeTile) * p.ntile);
  p.off_first = off;
  off = up256(off + sizeof(int) * p.nwg);
  p.off_qf = off;
  off = up256(off + size_t(lh) * p.ntile * p.qt * (d / 16) * 1024);
  p.off_qs = off;
  off = up256(off + size_t(lh) * p.ntile * M * 4);
  p.off_part = off;
  off = up256(off + size_t(lh) * (p.nwg + p.ntile) * M * d * 4);
  p.off_ml = off;
  p.bytes = up256(off + size_t(lh) * (p.nwg + p.ntile) * M * 8);
  return p;
}

// lh nwg is at most 3 CUs (one group of 32 rows; two: 2), or lh where that is more; a row's tiles are full but for its last one
double tree_plan_limit(int nl, int N, int B, int H, int Hq, int d) {
  const int grp = Hq / H;
  double most = 0;
  for (int qt = 1; qt <= 2; ++qt) {
    const int M = 32 * qt, heads = std::min(grp, M), nqc = (grp + heads - 1) / heads, tq = M / heads, rows = std::min(N, B);
    const double lh = double(nl) * H * nqc, ntile = std::min<double>(double(N) / tq + rows, N);
    const double parts = std::max(3.0 * cu_count(), lh) + lh * ntile;
    most = std::max(most, 256.0 * 8 + sizeof(TreeTile) * ntile + 12.0 * cu_count() + lh * ntile * (qt * (d / 16) * 1024.0 + M * 4.0) +
                              parts * M * (d * 4.0 + 8.0));
  }
  return most;
}

hipError_t launch_tree_attend(const ChunkDev& c0, const TreePlan& p, void* ws, const GaugeDev& G, const CodecDev& c, hipStream_t st) {
  TreeDev a;
  a.c = c0;
  a.c.tq = p.tq;
  a.c.heads = p.heads;
  a.c.nqc = p.nqc;
  a.c.ntile = p.ntile;
  a.bits = c.bits;
  a.qt = p.qt;
  a.nwg = p.nwg;
  char* base = static_cast<char*>(ws);
  a.line = reinterpret_cast<TreeLine*>(base);
  a.tiles = reinterpret_cast<TreeTile*>(base + p.off_tiles);
  a.first = reinterpret_cast<int*>(base + p.off_first);
  a.qf = reinterpret_cast<uint4*>(base + p.off_qf);
  a.qs = reinterpret_cast<float*>(base + p.off_qs);
  a.part = reinterpret_cast<float*>(base + p.off_part);
  a.ml = reinterpret_cast<float2*>(base + p.off_ml);
  const int d = a.c.q.d;
  const int64_t lh = int64_t(a.c.q.L) * a.c.kc.H * p.nqc, tiles = lh * p.ntile;
  if (tiles + 1 > 0x7fffffff || lh * p.nwg > 0x7fffffff) return hipErrorInvalidValue;
  GaugeDev g = G;
  void* args[] = {&a, &g};
  const void* fn = d == 64 ? (p.qt == 1 ? (const void*)tree_queries<64, 1> : (const void*)tree_queries<64, 2>)
                           : (p.qt == 1 ? (const void*)tree_queries<128, 1> : (const void*)tree_queries<128, 2>);
  hipError_t e = hipLaunchKernel(fn, dim3(unsigned(tiles + 1)), dim3(kPlanThreads), args, 0, st);
  if (e != hipSuccess) return e;
  const ChunkDev& b = a.c;
  const TreeRun r{b.kc.codes, b.vc.codes, b.kc.side, b.vc.side, b.pt.pages, b.mask, b.pos, b.err, a.line, a.tiles, a.first, a.qf, a.qs,
                  a.part, a.ml, b.l0, b.kc.H, b.nqc, b.heads, b.grp, c.n, b.pt.page_size, b.pt.max_pages, b.kc.B, b.words,
                  b.window, b.sinks, b.ntile, a.nwg};
  e = (d == 64 ? run_tree_attend_64 : run_tree_attend_128)(r, c.bits, p.qt, int(lh * p.nwg), st);
  if (e != hipSuccess) return e;
  const void* fj = d == 64 ? (p.qt == 1 ? (const void*)tree_join<64, 1> : (const void*)tree_join<64, 2>)
                           : (p.qt == 1 ? (const void*)tree_join<128, 1> : (const void*)tree_join<128, 2>);
  return hipLaunchKernel(fj, dim3(unsigned(tiles)), dim3(512), args, 0, st);
}

}  // namespace cg
