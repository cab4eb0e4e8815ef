// Keys of packed tokens turned by their positions, gauged and encoded to their slots on the matrix cores (the kernel:
// enc_mfma with kDestTurned).
#include "cg_enc_kernel.h"

namespace cg {

namespace {

template <int KS, int BITS>
const void* turned_by_nb(int nb) {
  switch (nb) {
    case 16: return (const void*)enc_mfma<3, KS, BITS, 16, kModeBU, 1, kDestTurned>;
    case 32: return (const void*)enc_mfma<3, KS, BITS, 32, kModeBU, 1, kDestTurned>;
    case 64: return (const void*)enc_mfma<3, KS, BITS, 64, kModeBU, 1, kDestTurned>;
  }
  return nullptr;
}
template <int KS>
const void* turned_by_bits(int bits, int nb) {
  switch (bits) {
    case 2: return turned_by_nb<KS, 2>(nb);
    case 3: return turned_by_nb<KS, 3>(nb);
    case 4: return turned_by_nb<KS, 4>(nb);
    case 6: return turned_by_nb<KS, 6>(nb);
    case 8: return turned_by_nb<KS, 8>(nb);
  }
  return nullptr;
}

}  // namespace

// Pairs in eights: of the two halves of the turned channels' granules, or of two neighbouring ones
bool turn_supported(const cg_rope_plan& plan) { return plan.d_rot % 16 == 0 && plan.d_rot <= kD; }

hipError_t launch_encode_turned(const ViewDev& Kn, int l0, const int* turn, const cg_rope_plan& rope, const int* slots,
                                const GaugeDev& G, const CodecDev& c, const CacheDev& kc, int* err, hipStream_t st) {
  TurnArgs m{};
  m.x = (char*)Kn.ptr;
  m.sl = Kn.sl; m.sh = Kn.sh; m.st = Kn.st;
  m.L = Kn.L; m.B = 1; m.H = Kn.H; m.T = m.tq = Kn.T;
  m.l0 = l0;
  for (int p = 0; p < 3; ++p) m.gp[p] = G.hi[p];
  m.g32 = G.f32; m.g = G.g; m.R = G.R; m.Hg = G.H;
  m.codes = kc.codes; m.side = kc.side;
  m.T_cap = kc.T_cap; m.cB = kc.B; m.cH = kc.H;
  m.err = err;
  m.pages = slots;
  m.turn = turn;
  m.plan = rope;
  const int ks = ksteps(G.g);
  const void* fn = ks == 2 ? turned_by_bits<2>(c.bits, c.n) : ks == 4 ? turned_by_bits<4>(c.bits, c.n) : turned_by_bits<8>(c.bits, c.n);
  if (!fn) return hipErrorInvalidValue;
  plan_at_most(m, Kn.L * Kn.H, Kn.T, fn, slot_tiles(kDestTurned));
  const int64_t nwg = (int64_t(m.nslices) * m.chunks + 7) / 8 * 8;
  if (nwg > INT32_MAX) return hipErrorInvalidValue;
  void* args[] = {&m};
  return hipLaunchKernel(fn, dim3(uint32_t(nwg)), dim3(kThreads), args, 0, st);
}

}  // namespace cg
