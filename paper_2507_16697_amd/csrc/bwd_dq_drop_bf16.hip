// Recompute backward with dropout, dQ part, bf16: launches of the kernel in bwd_dq_bf16_two_waves.h
// with it, at both head sizes.

#define RINGX_DROPOUT
#include "bwd_dq_bf16_two_waves.h"

namespace ringx {

hipError_t launch_bwd_dq_drop_bf16(const BwdArgs& a, const Drop& drop) {
  const QueryCut c = query_cut((a.Nq + 255) / 256 * a.BH, a.Nk, dq_cut_rule(a.d));
  if (a.d == 128) {
    if (c.ks == 4) return launch<128, 4, 8, 32>(a, drop);
    if (c.ks == 2) return launch<128, 2, 8, 64>(a, drop);
    return launch<128, 1, 8, 64>(a, drop);
  }
  if (c.half) return launch<64, 1, 4, 32>(a, drop);
  if (c.ks == 4) return launch<64, 4, 8, 64>(a, drop);
  if (c.ks == 2) return launch<64, 2, 8, 64>(a, drop);
  return launch<64, 1, 8, 64>(a, drop);
}

}  // namespace ringx
