// Sums of the parts that a split backward leaves: out = (out +) sum over s of part[s], in the order of s, what
// was there last.
// Bound by memory: the parts are read once, 16 bytes per lane.

#include "ringx_device.h"
#include "ringx_kernels.h"

namespace ringx {
namespace {

constexpr int kThreads = 256;

// blockIdx.y: which of the sums
__global__ __launch_bounds__(kThreads) void split_sum_kernel(SplitSums a) {
  const SplitSum& s = a.sum[blockIdx.y];
  const f32x4* part = reinterpret_cast<const f32x4*>(s.part);
  f32x4* out = reinterpret_cast<f32x4*>(s.out);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < s.n4;
       i += (int64_t)gridDim.x * kThreads) {
    f32x4 x = {};
#pragma unroll 8
    for (int p = 0; p < s.splits; ++p) x += part[(int64_t)p * s.n4 + i];
    out[i] = s.accumulate ? out[i] + x : x;
  }
}

}  // namespace

hipError_t launch_split_sums(const SplitSums& a, hipStream_t stream) {
  int64_t n4 = 0;
  for (int i = 0; i < a.count; ++i) n4 = n4 > a.sum[i].n4 ? n4 : a.sum[i].n4;
  const int64_t wgs = (n4 + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(split_sum_kernel, dim3((uint32_t)(wgs < 4096 ? wgs : 4096), (uint32_t)a.count),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ringx
