// Recompute backward, dK/dV part at head size 64: launches of the kernel in bwd_bf16_two_waves.h
// without dropout.

#include "bwd_bf16_two_waves.h"

namespace ringx {

// n = 128-key tiles of the launch.  Three shapes of the workgroup (us at 8192 queries; 8 waves x 64
// queries of a tile each / 8 waves x 32 / 4 waves x 32):
//   n =     96    128   192   256   266   384   390   474   512   626   1024  2048
//           110   119   123   133   258   236   267   276   260   377   515   1033
//           128   136   138   144   219   221   242   263   254   371   500   1009
//           96    110   126   141   190   205   290   296   282   326   526   1058
// With 32 queries per wave the kernel needs 127 registers and 65 KiB of LDS, so two workgroups share
// a CU and cover each other's barriers and loads: 2-3% faster where the chip is full (16384 queries
// and keys, 16 heads: at 1000 queries 187 -> 162).  64-key workgroups of 4 waves (138 registers, 49
// KiB, three per CU) end closer together where few tiles are left for the last round, and fill the
// chip earlier.  Between half a round and one round a CU has one workgroup anyway, and 64 queries
// per wave make fewer barriers.
hipError_t launch_bwd_dkdv_bf16_d64(const BwdArgs& a) {
  const int64_t n = a.BH / a.G * a.R * ds_tiles_per_chunk(a.Nk, a.R);
  const bool ragged = n > 256 && n < 1024 && (n - 1) % 256 < 128;
  if (n <= 128 || ragged) return launch<64, 4, 1>(a, NoDrop{});
  return n <= 256 ? launch<64, 8, 2>(a, NoDrop{}) : launch<64, 8, 1>(a, NoDrop{});
}

}  // namespace ringx
