// Recompute backward with dropout, dK/dV part, bf16: launches of the kernel in bwd_bf16_two_waves.h
// with it, at both head sizes.

#define RINGX_DROPOUT
#include "bwd_bf16_two_waves.h"

namespace ringx {

// n = 128-key tiles of the launch, those of every part of the sweep.  At d = 64, 64-key workgroups of
// 4 waves, three to a CU, where few tiles are left for the last round (n = 320: 368 us for the whole
// backward against 400 with 8 waves x 64 queries and 415 with 8 x 32) or the chip is not full, else 8 waves x 64 queries (n = 512: 320 against 352 and 326; n = 2048: 4430
// against 4590 and 4432), of whose two waves per SIMD each has the registers for the mask's
// constants: with 32 queries per wave, two workgroups to a CU, the 128 registers of a wave spill.
// At d = 128 8 waves fill a CU's SIMDs and 4 halve its tile: from more than half of the CUs on the
// former (n = 192: 80 against 102 us; n = 256: 259 against 338), below it the latter (n = 12: 33
// against 36).
hipError_t launch_bwd_dkdv_drop_bf16(const BwdArgs& a, const Drop& drop) {
  const int64_t whole = a.BH / a.G * ds_tiles_per_chunk(a.Nk, 1), n = whole * drop.splits;
  if (a.d == 128) return n <= 128 ? launch<128, 4, 1>(a, drop) : launch<128, 8, 1>(a, drop);
  return n <= 128 || ragged_last_round(whole) ? launch<64, 4, 1>(a, drop) : launch<64, 8, 2>(a, drop);
}

}  // namespace ringx
