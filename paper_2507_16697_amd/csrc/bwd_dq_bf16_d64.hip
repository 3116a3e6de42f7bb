// Recompute backward, dQ part at head size 64 and at 128 in launches that are cut: launches of the
// kernel in bwd_dq_bf16_two_waves.h without dropout.

#include "bwd_dq_bf16_two_waves.h"

namespace ringx {

hipError_t launch_bwd_dq_bf16_two_waves(const BwdArgs& a, const QueryCut& c) {
  if (a.d == 128) return c.ks == 4 ? launch<128, 4, 8, 32>(a, NoDrop{}) : launch<128, 2, 8, 64>(a, NoDrop{});
  if (c.half) return launch<64, 1, 4, 32>(a, NoDrop{});
  if (c.ks == 4) return launch<64, 4, 8, 64>(a, NoDrop{});
  if (c.ks == 2) return launch<64, 2, 8, 64>(a, NoDrop{});
  return launch<64, 1, 8, 64>(a, NoDrop{});
}

}  // namespace ringx
