// Matrix products of the linear layer in fp32 (gfx950): out[i][j] = sum over r of P(i, r) Q(j, r), then the
// epilogue of linear.h.  Operands of any stride and alignment.
//
// v_mfma_f32_32x32x2_f32 (full fp32 products and sums, 4096 flops in 64 cycles of a SIMD) with Q as its
// first operand: a lane holds one row i and four neighbouring j at a time.  Lane l has width index l % 32
// and, of 8 r, the four from 4 (l / 32) on; product e takes the e-th of them, so that an operand stored with r
// along its rows is one 16-byte load, one stored the other way four loads of 128 bytes of a row.
// A wave keeps BI x BJ blocks of 32 x 32; operands come from the caches without LDS, since a 64 x 64 tile
// needs 16 bytes per cycle and compute unit.  Loads are buffer loads from the tile's place on: what lies
// past the tensor reads as zero; r past R inside a row is masked in the last step.

#include "linear.h"

namespace ringx {
namespace {

__device__ __forceinline__ f32x16 mfma32f(float a, float b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

constexpr uint32_t kMostBytes = 0x7ffffff0u;

// One operand of a wave: B blocks of 32 of the width, 8 U of r at a time.
template <bool SLOW, int B, int U>
struct Feed {
  uint32_t off[B];
  int64_t base, left, step, row;   // bytes
  int g;

  __device__ __forceinline__ void start(const GemmIn& x, int64_t w0, int64_t r0, int lane) {
    g = lane >> 5;
    const int n = lane & 31;
    const int64_t at = SLOW ? r0 * x.ld + w0 : w0 * x.ld + r0;
    base = reinterpret_cast<int64_t>(uniform_ptr((const float*)x.p + at));
    left = 4 * ((x.rows - 1) * x.ld + x.cols - at);
    step = SLOW ? 32 * U * x.ld : 32 * U;
    row = 4 * x.ld;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if constexpr (SLOW) off[b] = (uint32_t)(16 * g * x.ld + 4 * (32 * b + n));
      else off[b] = (uint32_t)(4 * (min(w0 + 32 * b + n, x.rows - 1) - w0) * x.ld + 16 * g);
    }
  }
  __device__ __forceinline__ void load(f32x4 (&x)[U][B]) {
    const uint32_t bytes = left <= 0 ? 0u : left > (int64_t)kMostBytes ? kMostBytes : (uint32_t)left;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<void*>(uniform_ptr(reinterpret_cast<const void*>(base))), 0,
        __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if constexpr (SLOW) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[u][b][e] = __builtin_bit_cast(
                float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, off[b] + (8 * u + e) * (uint32_t)row, 0, 0));
        } else {
          x[u][b] = __builtin_bit_cast(
              f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off[b] + 32 * u, 0, 0));
        }
      }
    base += step, left -= step;
  }
  // zeros for r past the `rest` that there are
  __device__ __forceinline__ void mask(f32x4 (&x)[U][B], int rest) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = 8 * u + 4 * g + e < rest;
#pragma unroll
        for (int b = 0; b < B; ++b) x[u][b][e] = in ? x[u][b][e] : 0.f;
      }
  }
};

// A workgroup of four waves: 2 x 2 wave tiles (KS = 1), or one, whose r the waves split (KS = 4).
template <bool PS, bool QS, int B, int U, int KS>
__global__ __launch_bounds__(256, B == 2 ? 2 : 4) void gemm_f32_kernel(GemmArgs a) {
  constexpr int kTile = 32 * B * (KS == 1 ? 2 : 1), kStep = 8 * U;
  __shared__ float lds[KS == 1 ? 1 : (KS - 1) * 64 * 16 * B * B];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ti = (uint32_t)((a.I + kTile - 1) / kTile), tj = (uint32_t)((a.J + kTile - 1) / kTile);
  constexpr uint32_t kGroup = 8;
  uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t split = id / (ti * tj);
  id -= split * ti * tj;
  const uint32_t g0 = id / (kGroup * tj) * kGroup, gn = min(kGroup, ti - g0);
  id -= g0 * tj;
  int64_t i0 = (int64_t)(g0 + id % gn) * kTile, j0 = (int64_t)(id / gn) * kTile;
  if (KS == 1) i0 += 32 * B * (wave >> 1), j0 += 32 * B * (wave & 1);
  const int ks = KS == 1 ? 0 : wave;

  const int64_t steps = (a.R + kStep - 1) / kStep, parts = (int64_t)a.splits * KS;
  const int64_t part = (int64_t)split * KS + ks;
  const int64_t s0 = steps * part / parts, s1 = steps * (part + 1) / parts;
  f32x16 acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = f32x16{};
  if (s0 < s1 && i0 < a.I && j0 < a.J) {
    Feed<PS, B, U> fp;
    Feed<QS, B, U> fq;
    fp.start(a.P, i0, s0 * kStep, lane);
    fq.start(a.Q, j0, s0 * kStep, lane);
    f32x4 p[U][B], q[U][B];
    fp.load(p);
    fq.load(q);
    for (int64_t s = s0; s < s1; ++s) {
      f32x4 pn[U][B], qn[U][B];
      if (s + 1 < s1) {
        fp.load(pn);
        fq.load(qn);
      }
      const int64_t rest = a.R - s * kStep;
      if (rest < kStep) {
        cold_path();
        fp.mask(p, (int)rest);
        fq.mask(q, (int)rest);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < B; ++i)
#pragma unroll
            for (int j = 0; j < B; ++j) acc[i][j] = mfma32f(q[u][j][e], p[u][i][e], acc[i][j]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < B; ++b) p[u][b] = pn[u][b], q[u][b] = qn[u][b];
    }
  }
  if constexpr (KS > 1) {
    // the waves' sums, in their order
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            lds[(((wave - 1) * B * B + i * B + j) * 16 + r) * 64 + lane] = acc[i][j][r];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < KS - 1; ++w)
#pragma unroll
      for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            acc[i][j][r] += lds[((w * B * B + i * B + j) * 16 + r) * 64 + lane];
  }
  GemmOut o = a.o;
  const bool vec = a.J % 4 == 0 && o.d % 4 == 0;
  if (a.splits > 1) {
    o = GemmOut{};
    o.out = a.part + split * a.I * a.J, o.J = a.J, o.f32 = true;
  }
#pragma unroll
  for (int bi = 0; bi < B; ++bi) {
    const int64_t i = i0 + 32 * bi + (lane & 31);
#pragma unroll
    for (int bj = 0; bj < B; ++bj)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t j = j0 + 32 * bj + 8 * r + 4 * (lane >> 5);
        const int inside = (int)max((int64_t)0, min((int64_t)4, a.J - j));
        if (i >= a.I || inside == 0) continue;
        float b[4], x[4] = {acc[bi][bj][4 * r], acc[bi][bj][4 * r + 1], acc[bi][bj][4 * r + 2],
                            acc[bi][bj][4 * r + 3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = o.bias && e < inside ? o.bias[j + e] : 0.f;
        if (vec) finish<4, true, float>(o, i, j, 4, b, x);
        else finish<4, false, float>(o, i, j, inside, b, x);
      }
  }
}

template <bool PS, bool QS, int B, int U, int KS>
hipError_t launch(const GemmArgs& a) {
  constexpr int kTile = 32 * B * (KS == 1 ? 2 : 1);
  const int64_t tiles = ((a.I + kTile - 1) / kTile) * ((a.J + kTile - 1) / kTile) * a.splits;
  hipLaunchKernelGGL((gemm_f32_kernel<PS, QS, B, U, KS>), dim3((uint32_t)tiles), dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

template <int B, int U, int KS>
hipError_t by_layout(const GemmArgs& a) {
  if (a.p_slow) return launch<true, true, B, U, KS>(a);
  return a.q_slow ? launch<false, true, B, U, KS>(a) : launch<false, false, B, U, KS>(a);
}

}  // namespace

hipError_t launch_gemm_f32(const GemmArgs& a) {
  return gemm_f32_large(a.I, a.J) ? by_layout<2, 2, 1>(a) : by_layout<1, 4, 4>(a);
}

}  // namespace ringx
