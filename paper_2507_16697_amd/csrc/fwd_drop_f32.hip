// Attention forward with dropout, fp32: launches of the kernel in fwd_f32_kernel.h with it.

#define RINGX_DROPOUT
#include "fwd_f32_kernel.h"

namespace ringx {

hipError_t launch_fwd_drop_f32(const FwdArgs& a, FwdMode mode, const Drop& drop) {
  return launch_any(a, mode, drop);
}

}  // namespace ringx
