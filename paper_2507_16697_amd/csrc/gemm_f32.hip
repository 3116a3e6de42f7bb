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
  uint32_t off[B], row;        // bytes
  int64_t base, left, step;
  int g;

  // sizes fit 32 bits
  __device__ __forceinline__ void start(const GemmIn& x, uint32_t w0, uint32_t r0, int lane) {
    g = lane >> 5;
    const uint32_t n = lane & 31, rows = (uint32_t)x.rows, ld = (uint32_t)x.ld;
    const int64_t at = SLOW ? (int64_t)r0 * ld + w0 : (int64_t)w0 * ld + r0;
    base = reinterpret_cast<int64_t>(uniform_ptr((const float*)x.p + at));
    left = 4 * ((int64_t)(rows - 1) * ld + (uint32_t)x.cols - at);
    step = SLOW ? 32 * U * (int64_t)ld : 32 * U;
    row = 4 * ld;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if constexpr (SLOW) off[b] = 16 * g * ld + 4 * (32 * b + n);
      else off[b] = 4 * (min(w0 + 32 * b + n, rows - 1) - w0) * ld + 16 * g;
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
                float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, off[b] + (8 * u + e) * row, 0, 0));
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

// A workgroup of four waves: 2 x 2 wave tiles (KS = 1), or one of 32 x 32, whose r the waves split (KS = 4).
template <bool PS, bool QS, int B, int U, int KS>
__global__ __launch_bounds__(256, B == 2 ? 2 : 4) void gemm_f32_kernel(GemmArgs a) {
  constexpr uint32_t kTile = 32 * B * (KS == 1 ? 2 : 1), kStep = 8 * U;
  static_assert(KS == 1 || B == 1, "one block of four waves");
  // a wave's block of 32 x 32, by lane and register, or by row and column
  constexpr int kBlock = 64 * 17;
  __shared__ float lds[4 * kBlock];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t I = (uint32_t)a.I, J = (uint32_t)a.J, R = (uint32_t)a.R;
  const uint32_t ti = (I + kTile - 1) / kTile, tj = (J + kTile - 1) / kTile;
  constexpr uint32_t kGroup = 8;
  uint32_t id = xcd_remap(blockIdx.x, gridDim.x), split = 0;
  if (a.splits > 1) {
    split = id / (ti * tj);
    id -= split * ti * tj;
  }
  const uint32_t g0 = id / (kGroup * tj) * kGroup, gn = min(kGroup, ti - g0);
  id -= g0 * tj;
  uint32_t i0 = (g0 + id % gn) * kTile, j0 = (id / gn) * kTile;
  if (KS == 1) i0 += 32 * B * (wave >> 1), j0 += 32 * B * (wave & 1);

  const uint32_t steps = (R + kStep - 1) / kStep, parts = (uint32_t)a.splits * KS;
  const uint32_t part = split * KS + (KS == 1 ? 0 : wave);
  uint32_t s0 = 0, s1 = steps;
  if (parts > 1) s0 = (uint32_t)((uint64_t)steps * part / parts), s1 = (uint32_t)((uint64_t)steps * (part + 1) / parts);
  f32x16 acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = f32x16{};
  if (s0 < s1 && i0 < I && j0 < J) {
    Feed<PS, B, U> fp;
    Feed<QS, B, U> fq;
    fp.start(a.P, i0, s0 * kStep, lane);
    fq.start(a.Q, j0, s0 * kStep, lane);
    f32x4 p[U][B], q[U][B];
    fp.load(p);
    fq.load(q);
    for (uint32_t s = s0; s < s1; ++s) {
      f32x4 pn[U][B], qn[U][B];
      if (s + 1 < s1) {
        fp.load(pn);
        fq.load(qn);
      }
      const uint32_t rest = R - s * kStep;
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
  GemmOut o = a.o;
  const bool vec = J % 4 == 0 && o.d % 4 == 0;
  if (a.splits > 1) {
    o = GemmOut{};
    o.out = a.part + split * a.I * a.J, o.J = a.J, o.f32 = true;
  }
  const auto bias = [&](uint32_t j) { return o.bias && j < J ? o.bias[j] : 0.f; };
  if constexpr (KS > 1) {
    // the waves' sums in their order; then all of them end the block, neighbouring columns in neighbouring
    // lanes
#pragma unroll
    for (int r = 0; r < 16; ++r) lds[wave * kBlock + lane * 17 + r] = acc[0][0][r];
    __syncthreads();
    const auto sum = [&](uint32_t i, uint32_t j) {
      const uint32_t at = (i + 32 * (j >> 2 & 1)) * 17 + 4 * (j >> 3) + (j & 3);
      float t = lds[at];
#pragma unroll
      for (int w = 1; w < KS; ++w) t += lds[w * kBlock + at];
      return t;
    };
    if (vec) {
      const uint32_t i = threadIdx.x / 8, j = threadIdx.x % 8 * 4;
      float x[4], b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = sum(i, j + e), b[e] = bias(j0 + j + e);
      if (i0 + i < I && j0 + j < J) finish<4, true, float>(o, i0 + i, j0 + j, 4, b, x);
    } else {
      const uint32_t j = threadIdx.x % 32;
      float b[1] = {bias(j0 + j)};
#pragma unroll 1
      for (uint32_t i = threadIdx.x / 32; i < 32; i += 8) {
        float x[1] = {sum(i, j)};
        if (i0 + i < I && j0 + j < J) finish<1, false, float>(o, i0 + i, j0 + j, 1, b, x);
      }
    }
    return;
  }
#pragma unroll
  for (int bi = 0; bi < B; ++bi)
#pragma unroll
    for (int bj = 0; bj < B; ++bj) {
      const uint32_t ib = i0 + 32 * bi, jb = j0 + 32 * bj;
      if (vec) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t i = ib + (lane & 31), j = jb + 8 * r + 4 * (lane >> 5);
          float b[4], x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = acc[bi][bj][4 * r + e], b[e] = bias(j + e);
          if (i < I && j < J) finish<4, true, float>(o, i, j, 4, b, x);
        }
      } else {
        float* const stage = lds + wave * kBlock;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          stage[(lane & 31) * 33 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4] = acc[bi][bj][r];
        __builtin_amdgcn_wave_barrier();
        const uint32_t j = lane & 31;
        float b[1] = {bias(jb + j)};
#pragma unroll 1
        for (uint32_t i = lane >> 5; i < 32; i += 2) {
          float x[1] = {stage[i * 33 + j]};
          if (ib + i < I && jb + j < J) finish<1, false, float>(o, ib + i, jb + j, 1, b, x);
        }
        __builtin_amdgcn_wave_barrier();
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
  return gemm_f32_large(a.I, a.J) ? by_layout<2, 4, 1>(a) : by_layout<1, 4, 4>(a);
}

}  // namespace ringx
