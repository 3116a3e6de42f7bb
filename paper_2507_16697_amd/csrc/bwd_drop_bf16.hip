// Recompute backward with dropout, dK/dV part, bf16: launches of the kernel in bwd_bf16_two_waves.h
// with it, at both head sizes.

#include "bwd_bf16_two_waves.h"

namespace ringx {

hipError_t launch_bwd_dkdv_drop_bf16(const BwdArgs& a, const Drop& drop) {
  const int64_t n = a.BH / a.G * ds_tiles_per_chunk(a.Nk, 1);
  const bool ragged = n > 256 && n < 1024 && (n - 1) % 256 < 128;
  if (a.d == 128) return n <= 128 ? launch<128, 4, 1>(a, drop) : launch<128, 8, 1>(a, drop);
  if (n <= 128 || ragged) return launch<64, 4, 1>(a, drop);
  return n <= 256 ? launch<64, 8, 2>(a, drop) : launch<64, 8, 1>(a, drop);
}

}  // namespace ringx
