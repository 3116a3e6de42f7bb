// Recompute backward with dropout, fp32: launches of the kernel in bwd_f32_kernel.h with it.

#define RINGX_DROPOUT
#include "bwd_f32_kernel.h"

namespace ringx {

hipError_t launch_bwd_drop_f32(const BwdArgs& a, const Drop& drop) {
  return launch_any(a, true, true, drop);
}

}  // namespace ringx
