// Matrix-core codec kernels for bf16 caches with head dimension 128 and the block-uniform
// backend (the configuration the paper's Llama-class KV caches take).
//
// The gauge (section 3: z = G_{l,s,h,r} x per channel group) is a dense contraction over the
// channel axis, so it runs on the gfx950 matrix cores with v_mfma_f32_32x32x16_bf16.  The
// input x is exact in bf16; the binary32 gauge enters as kNP bf16 planes G0 + G1 (+ G2) of
// its split (the gauge buffer holds three), each multiplied on the matrix core with a
// binary32 accumulator.  Two planes carry 16 significant bits of every entry (entry error at
// most 2^-16 relative), which keeps z within a few 1e-6 of the binary32 gauge per group,
// inside the 1e-5 gauge tolerance, at two thirds of the matrix-core work of three planes.
//
// Work split: a workgroup of four wave64s owns a range of 32-token tiles of one
// (layer, batch, head) slice; wave w computes output channels [32w, 32w+32) (one 32-row MFMA
// tile) for the tile's 32 tokens.  The wave keeps its 32 rows of every split plane in VGPRs
// for the whole range, so the matrix core never re-reads G.  Output rows are permuted so
// that lane (token n, half hc) ends up with the 16 consecutive channels 32w + 16hc + [0, 16):
// its codes form one contiguous stretch of the packed row.  Tokens are staged through LDS
// with an XOR swizzle of the 16-byte granules of each 256-byte row, so the B-operand reads
// (lane n reads granule j of row n) hit distinct banks.
//
// Encode epilogue (section 4.3 block-uniform): block minimum / maximum in-lane, across the
// two lane halves (n = 32) and across the wave pair through LDS (n = 64); binary16 side
// information; binary32 quantisation without contraction; LSB-first packing; stores.
//
#include "cg_enc_kernel.h"

namespace cg {

namespace {

// Split planes of the gauge on the matrix core.  Decoding takes two (16 significant bits per
// entry: a few 1e-6 of the group norm).  Encoding takes two up to 4-bit codes and three
// above: a finer grid turns the same z error into more codes moved across a rounding
// boundary (with two planes about 3e-5 of 4-bit codes but 1.4e-4 of 6-bit codes move, against
// the 1e-4 budget).
constexpr int enc_planes(int bits) { return bits >= 6 ? 3 : 2; }

template <int KS, int BITS, int NB>
void* enc_kernel(int mode, int bt) {
  if (mode == kModePass) return (void*)enc_mfma<kNP, KS, 8, 64, kModePass>;
  if (mode == kModeZfp) return NB == 64 ? (void*)enc_mfma<kNP, KS, BITS, 64, kModeZfp> : nullptr;
  if (mode == kModeKeys) return (void*)enc_mfma<enc_planes(BITS), KS, BITS, 32, kModeKeys>;
  if constexpr (NB >= 64) {
    if (bt == 16) return (void*)enc_mfma<enc_planes(BITS), KS, BITS, NB, kModeBU, 16>;
  }
  if constexpr (NB <= 64) {
    if (bt == 1) return (void*)enc_mfma<enc_planes(BITS), KS, BITS, NB, kModeBU>;
  }
  return nullptr;
}

// Paged caches take three planes at every width: their encoder was the binary32 FMA chain, and three
// planes (24 significant bits of every entry) keep z closer to the binary64 product than that chain does
// (relative error 1.2e-7 against 2.0e-7 at g = 128, 0.7e-7 against 1.0e-7 at g = 32).  8 layers x 4 rows x
// 8 heads x 2000 tokens in 256-position pages, g = 128, 4 bits: 1058 us per tensor on the vector ALU, 236
// on the binary32 matrix cores (the general kernel, which other shapes keep), 70 here.
constexpr int kModePaged = 4, kModeSlots = 5;

template <int KS, int BITS>
void* enc_by_nb(int nb, int mode, int bt) {
  if (mode == kModePaged || mode == kModeSlots) {
    const bool slots = mode == kModeSlots;
    switch (nb) {
      case 16: return slots ? (void*)enc_mfma<3, KS, BITS, 16, kModeBU, 1, kDestSlots> : (void*)enc_mfma<3, KS, BITS, 16, kModeBU, 1, kDestPages>;
      case 32: return slots ? (void*)enc_mfma<3, KS, BITS, 32, kModeBU, 1, kDestSlots> : (void*)enc_mfma<3, KS, BITS, 32, kModeBU, 1, kDestPages>;
      case 64: return slots ? (void*)enc_mfma<3, KS, BITS, 64, kModeBU, 1, kDestSlots> : (void*)enc_mfma<3, KS, BITS, 64, kModeBU, 1, kDestPages>;
    }
    return nullptr;
  }
  switch (nb) {
    case 16: return enc_kernel<KS, BITS, 16>(mode, bt);
    case 32: return enc_kernel<KS, BITS, 32>(mode, bt);
    case 64: return enc_kernel<KS, BITS, 64>(mode, bt);
    case 128: return enc_kernel<KS, BITS, 128>(mode, bt);
  }
  return nullptr;
}

template <int KS>
void* enc_by_bits(int bits, int nb, int mode, int bt) {
  switch (bits) {
    case 2: return enc_by_nb<KS, 2>(nb, mode, bt);
    case 3: return enc_by_nb<KS, 3>(nb, mode, bt);
    case 4: return enc_by_nb<KS, 4>(nb, mode, bt);
    case 6: return enc_by_nb<KS, 6>(nb, mode, bt);
    case 8: return enc_by_nb<KS, 8>(nb, mode, bt);
  }
  return nullptr;
}

const void* enc_of(int g, int bits, int nb, int mode, int bt) {
  switch (ksteps(g)) {
    case 2: return enc_by_bits<2>(bits, nb, mode, bt);
    case 4: return enc_by_bits<4>(bits, nb, mode, bt);
    case 8: return enc_by_bits<8>(bits, nb, mode, bt);
  }
  return nullptr;
}

}  // namespace

bool mfma_encode_supported(const ViewDev& X, const GaugeDev& G, const CodecDev& c, bool paged) {
  if (!X.bf16 || X.d != kD || !group_ok(G.g)) return false;
  if (paged && c.backend != CG_BACKEND_BLOCK_UNIFORM) return false;  // the error-free backend: general kernels
  if (c.backend == CG_BACKEND_PASSTHROUGH) return true;
  if (c.backend == CG_BACKEND_ZFP) return bits_ok(c.bits);
  if (c.backend == CG_BACKEND_KIVI)
    return bits_ok(c.bits) && c.kg == kTok && (c.kvc == 16 || c.kvc == 32 || c.kvc == 64) && c.win % kTok == 0;
  if (c.backend != CG_BACKEND_BLOCK_UNIFORM || !bits_ok(c.bits)) return false;
  if (c.bt == 16) return c.n == 64 || c.n == 128;  // token-channel tiles
  return c.bt == 1 && (c.n == 16 || c.n == 32 || c.n == 64);
}

hipError_t launch_encode_mfma(int s, const ViewDev& X, int l0, const GaugeDev& G, const CodecDev& c,
                              const CacheDev& k, int t0, int tq, int* err, hipStream_t st, const PageDev& pt) {
  if (X.T == 0) return hipSuccess;
  MfmaArgs m{};
  m.x = (char*)X.ptr;
  m.sl = X.sl; m.sb = X.sb; m.sh = X.sh; m.st = X.st;
  m.L = X.L; m.B = X.B; m.H = X.H; m.T = X.T;
  m.l0 = l0; m.s = s; m.t0 = t0;
  for (int p = 0; p < 3; ++p) m.gp[p] = G.hi[p];
  m.g32 = G.f32; m.g = G.g; m.R = G.R; m.Hg = G.H;
  m.codes = k.codes; m.side = k.side; m.T_cap = k.T_cap; m.cB = k.B; m.cH = k.H;
  m.err = err;
  const bool pass = c.backend == CG_BACKEND_PASSTHROUGH, kivi = c.backend == CG_BACKEND_KIVI;
  const bool zfp = c.backend == CG_BACKEND_ZFP;
  const bool tiles = c.backend == CG_BACKEND_BLOCK_UNIFORM && c.bt > 1;
  m.tq = kivi || tiles ? tq : X.T;
  m.ring = k.ring;
  m.ring_slots = kivi ? c.win + c.kg : (tiles ? c.bt : 0);
  m.pages = pt.pages;
  m.max_pages = pt.max_pages;
  const int mode = pt.pages ? kModePaged : pass ? kModePass : (zfp ? kModeZfp : (kivi && s == 0 ? kModeKeys : kModeBU));
  const int nb = pass || zfp ? 64 : (kivi ? c.kvc : c.n), bits = pass ? 8 : c.bits, bt = tiles ? c.bt : 1;
  const void* fn = enc_of(G.g, bits, nb, mode, bt);
  if (!fn) return hipErrorInvalidValue;
  plan(m, X.L * X.B * X.H, X.T, fn);
  const int nwg = ((m.nslices * m.chunks + 7) / 8) * 8;
  void* args[] = {&m};
  return hipLaunchKernel(fn, dim3(nwg), dim3(kThreads), args, 0, st);
}

hipError_t launch_encode_slots(const ViewDev& Kn, const ViewDev& Vn, int l0, const int* slots, const GaugeDev& G,
                               const CodecDev& c, const CacheDev& kc, const CacheDev& vc, int* err, hipStream_t st,
                               const int* turn) {
  MfmaArgs m{};
  m.x = (char*)Kn.ptr;
  m.sl = Kn.sl; m.sh = Kn.sh; m.st = Kn.st;
  m.v.x = (char*)Vn.ptr;
  m.v.sl = Vn.sl; m.v.sh = Vn.sh; m.v.st = Vn.st;
  m.L = Kn.L; m.B = 1; m.H = Kn.H; m.T = m.tq = Kn.T;
  m.l0 = l0;
  for (int p = 0; p < 3; ++p) m.gp[p] = G.hi[p];
  m.g32 = G.f32; m.g = G.g; m.R = G.R; m.Hg = G.H;
  m.codes = kc.codes; m.side = kc.side; m.v.codes = vc.codes; m.v.side = vc.side;
  m.T_cap = kc.T_cap; m.cB = kc.B; m.cH = kc.H;
  m.err = err;
  m.pages = slots;
  m.turn = turn;
  if (turn) {
    m.s = 1;
    m.x = m.v.x; m.sl = m.v.sl; m.sh = m.v.sh; m.st = m.v.st;
    m.codes = m.v.codes; m.side = m.v.side;
  }
  const void* fn = enc_of(G.g, c.bits, c.n, kModeSlots, 1);
  if (!fn) return hipErrorInvalidValue;
  plan_at_most(m, (turn ? 1 : 2) * Kn.L * Kn.H, Kn.T, fn, slot_tiles(kDestSlots));
  const int64_t nwg = (int64_t(m.nslices) * m.chunks + 7) / 8 * 8;
  if (nwg > INT32_MAX) return hipErrorInvalidValue;
  void* args[] = {&m};
  return hipLaunchKernel(fn, dim3(uint32_t(nwg)), dim3(kThreads), args, 0, st);
}

}  // namespace cg
