// Matrix products of the linear layer in fp32 (gfx950): out[i][j] = sum over r of P(i, r) Q(j, r), then the
// epilogue of linear.h.
//
// v_mfma_f32_32x32x2_f32 (full fp32 products and sums, 4096 flops in 64 cycles of a SIMD) with Q as its
// first operand: a lane holds one row i and four neighbouring j at a time.  Lane l has width index l % 32
// and, of 8 r, the four from 4 (l / 32) on; product e takes the e-th of them, so that an operand stored with r
// along its rows is one 16-byte read, one stored the other way four reads of 128 bytes of a row.
//
// Tiles of 128 x 128 or 64 x 64 through LDS (gemm_feed.h), a quarter to a wave.  Where those are few: blocks of
// 32 x 32, whose r the four waves of a workgroup split, from the caches without LDS; these take operands of any
// stride and alignment.

#include "gemm_feed.h"
#include "linear.h"

namespace ringx {
namespace {

__device__ __forceinline__ f32x16 mfma32f(float a, float b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// One operand of a wave: 32 of the width, 8 U of r at a time.
template <bool SLOW, int U>
struct Direct {
  uint32_t off, row;           // bytes
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
    if constexpr (SLOW) off = 16 * g * ld + 4 * n;
    else off = 4 * (min(w0 + n, rows - 1) - w0) * ld + 16 * g;
  }
  __device__ __forceinline__ void load(f32x4 (&x)[U]) {
    const uint32_t bytes = left <= 0 ? 0u : left > (int64_t)kMostBytes ? kMostBytes : (uint32_t)left;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<void*>(uniform_ptr(reinterpret_cast<const void*>(base))), 0,
        __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (SLOW) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[u][e] = __builtin_bit_cast(
              float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, off + (8 * u + e) * row, 0, 0));
      } else {
        x[u] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 32 * u, 0, 0));
      }
    }
    base += step, left -= step;
  }
  // zeros for r past the `rest` that there are
  __device__ __forceinline__ void mask(f32x4 (&x)[U], int rest) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = 8 * u + 4 * g + e < rest ? x[u][e] : 0.f;
  }
};

// One block of 32 x 32 whose r four waves (and, a.splits > 1, as many workgroups) share.
constexpr int kWaves = 4, kU = 4;
constexpr uint32_t kSide = 32, kStep = 8 * kU;

template <bool PS, bool QS>
__device__ __forceinline__ void small_product(const GemmArgs& a, uint32_t id, uint32_t wgs, float* lds) {
  constexpr int kBlock = 64 * 17;   // a wave's values by lane and register
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t I = (uint32_t)a.I, J = (uint32_t)a.J, R = (uint32_t)a.R;
  const uint32_t ti = (I + kSide - 1) / kSide, tj = (J + kSide - 1) / kSide;
  constexpr uint32_t kGroup = 8;
  id = xcd_remap(id, wgs);
  uint32_t split = 0;
  if (a.splits > 1) {
    split = id / (ti * tj);
    id -= split * ti * tj;
  }
  const uint32_t g0 = id / (kGroup * tj) * kGroup, gn = min(kGroup, ti - g0);
  id -= g0 * tj;
  const uint32_t i0 = (g0 + id % gn) * kSide, j0 = (id / gn) * kSide;

  const uint32_t steps = (R + kStep - 1) / kStep, parts = (uint32_t)a.splits * kWaves;
  const uint32_t part = split * kWaves + wave;
  const uint32_t s0 = (uint32_t)((uint64_t)steps * part / parts), s1 = (uint32_t)((uint64_t)steps * (part + 1) / parts);
  f32x16 acc = {};
  if (s0 < s1) {
    Direct<PS, kU> fp;
    Direct<QS, kU> fq;
    fp.start(a.P, i0, s0 * kStep, lane);
    fq.start(a.Q, j0, s0 * kStep, lane);
    f32x4 p[kU], q[kU];
    fp.load(p);
    fq.load(q);
    for (uint32_t s = s0; s < s1; ++s) {
      f32x4 pn[kU], qn[kU];
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
      for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = mfma32f(q[u][e], p[u][e], acc);
#pragma unroll
      for (int u = 0; u < kU; ++u) p[u] = pn[u], q[u] = qn[u];
    }
  }
  GemmOut o = a.o;
  const bool vec = J % 4 == 0 && o.d % 4 == 0;
  if (a.splits > 1) {
    o = GemmOut{};
    o.out = a.part + split * a.I * a.J, o.J = a.J, o.f32 = true;
  }
  const auto bias = [&](uint32_t j) { return o.bias && j < J ? o.bias[j] : 0.f; };
  // the waves' sums in their order; then all of them end the block, neighbouring columns in neighbouring
  // lanes
#pragma unroll
  for (int r = 0; r < 16; ++r) lds[wave * kBlock + lane * 17 + r] = acc[r];
  __syncthreads();
  const auto sum = [&](uint32_t i, uint32_t j) {
    const uint32_t at = (i + 32 * (j >> 2 & 1)) * 17 + 4 * (j >> 3) + (j & 3);
    float t = lds[at];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) t += lds[w * kBlock + at];
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
}
constexpr int kSmallLds = kWaves * 64 * 17;

// Fragments of a tile in LDS: 32 of the width x 8 of r.
template <bool SLOW, int W>
struct Frags {
  using F = Feed<float, SLOW, W, 256>;
  static constexpr int kBlocks = W / 64, kRow = 4 * W;   // of a wave; bytes of a slow row
  int off[SLOW ? kBlocks : 4];
  __device__ __forceinline__ void start(int w0, int lane) {   // w0: the wave's first of the tile
    const int n = lane & 31, g = lane >> 5;
    if constexpr (!SLOW) {
#pragma unroll
      for (int u = 0; u < 4; ++u) off[u] = (w0 + n) * 128 + (((2 * u + g) ^ F::swz(w0 + n)) << 4);
    } else {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int col = w0 + 32 * b + n;
        off[b] = 4 * g * kRow + (((col >> 2) ^ F::swz(4 * g)) << 4) + (col & 3) * 4;
      }
    }
  }
  __device__ __forceinline__ f32x4 get(const char* tile, int u, int b) const {
    if constexpr (!SLOW) {
      return *reinterpret_cast<const f32x4*>(tile + off[u] + b * 32 * 128);
    } else {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const float*>(tile + off[b] + (8 * u + e) * kRow);
      return x;
    }
  }
};

// Tiles of W x W, four waves of W / 2 x W / 2 in blocks of 32 x 32.  Bound by the matrix cores (W = 128, two
// workgroups to a compute unit), or by the latency of a step (W = 64, four).
constexpr int tile_lds(int W) { return 4 * W * 128; }   // two buffers of two operands

template <bool PS, bool QS, int W>
__device__ __forceinline__ void tile_product(const GemmArgs& a, uint32_t id, uint32_t wgs, char* lds) {
  constexpr int kP = W * 128, kStage = 2 * kP, BK = 32, B = W / 64, kProducts = 4 * B * B;
  const uint32_t lbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / 2, wj = wave % 2;
  const uint32_t I = (uint32_t)a.I, J = (uint32_t)a.J;
  uint32_t i_tile, j_tile;
  place(xcd_remap(id, wgs), (I + W - 1) / W, (J + W - 1) / W, i_tile, j_tile);
  const uint32_t i0 = i_tile * W, j0 = j_tile * W;
  Feed<float, PS, W, 256> fp;
  Feed<float, QS, W, 256> fq;
  fp.start(a.P, i0, 0, tid);
  fq.start(a.Q, j0, 0, tid);
  Frags<PS, W> rp;
  Frags<QS, W> rq;
  rp.start(wi * (W / 2), lane);
  rq.start(wj * (W / 2), lane);
  const uint32_t wdst = (uint32_t)__builtin_amdgcn_readfirstlane(lbase + wave * 1024);
  f32x16 acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = f32x16{};

  // Unit T - 1's products (8 of r), beside them the reads of unit T of the step in `buf` and a later step's
  // loads.
  f32x4 p[2][B], q[2][B];
  auto unit = [&](auto t, uint32_t buf, auto feed, auto loads) {
    constexpr int T = decltype(t)::value, L = decltype(loads)::value, S = T & 1;
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
#pragma unroll
      for (int u = i * L / kProducts; u < (i + 1) * L / kProducts; ++u) feed(u);
#pragma unroll
      for (int f = i * 2 * B / kProducts; f < (i + 1) * 2 * B / kProducts; ++f) {
        if (f % 2 == 0) q[S][f / 2] = rq.get(lds + buf + kP, T, f / 2);
        else p[S][f / 2] = rp.get(lds + buf, T, f / 2);
      }
      const int e = i / (B * B), bi = i / B % B, bj = i % B;
      acc[bi][bj] = mfma32f(q[S ^ 1][bj][e], p[S ^ 1][bi][e], acc[bi][bj]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto nothing = [](int) {};
  using std::integral_constant;
  typedef integral_constant<int, 0> kNone;
  typedef integral_constant<int, Feed<float, PS, W, 256>::kLoads> kLoads;
  int rest = (int)a.R;
  const int steps = (rest + BK - 1) / BK;
  fp.all(wdst, rest);
  fq.all(wdst + kP, rest);
  rest -= BK;
  fp.all(wdst + kStage, rest);
  wait_vmem<kLoads::value>();
  __syncthreads();
#pragma unroll
  for (int b = 0; b < B; ++b) q[0][b] = rq.get(lds + kP, 0, b), p[0][b] = rp.get(lds, 0, b);
  uint32_t buf = 0;
  for (int s = steps; s > 0; --s) {
    fq.begin(rest);
    unit(integral_constant<int, 1>{}, buf, [&](int u) { fq.load(u, wdst + kStage - buf + kP); }, kLoads{});
    rest -= BK;
    unit(integral_constant<int, 2>{}, buf, nothing, kNone{});
    unit(integral_constant<int, 3>{}, buf, nothing, kNone{});
    wait_vmem_all();
    __syncthreads();
    fp.begin(rest);
    buf = kStage - buf;
    unit(integral_constant<int, 0>{}, buf, [&](int u) { fp.load(u, wdst + kStage - buf); }, kLoads{});
  }
  wait_vmem_all();
  __syncthreads();

  const GemmOut& o = a.o;
  const bool vec = J % 4 == 0 && o.d % 4 == 0;
  const auto bias = [&](uint32_t j) { return o.bias && j < J ? o.bias[j] : 0.f; };
  float* const stage = reinterpret_cast<float*>(lds) + wave * 32 * 33;
#pragma unroll
  for (int bi = 0; bi < B; ++bi)
#pragma unroll
    for (int bj = 0; bj < B; ++bj) {
      const uint32_t ib = i0 + wi * (W / 2) + 32 * bi, jb = j0 + wj * (W / 2) + 32 * bj;
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
        // through LDS, a lane one column of row after row
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

// SIDE: of a tile, or 32 for small blocks
template <bool PS, bool QS, int SIDE>
__device__ __forceinline__ void product(const GemmArgs& a, uint32_t id, uint32_t wgs, char* lds) {
  if constexpr (SIDE == 32) small_product<PS, QS>(a, id, wgs, reinterpret_cast<float*>(lds));
  else tile_product<PS, QS, SIDE>(a, id, wgs, lds);
}
template <int SIDE>
constexpr int kLds = SIDE == 32 ? kSmallLds * 4 : tile_lds(SIDE);
template <int SIDE>
constexpr int kPerUnit = SIDE == 128 ? 2 : 4;   // workgroups of a compute unit

template <bool PS, bool QS, int SIDE>
__global__ __launch_bounds__(256, kPerUnit<SIDE>) void gemm_f32_kernel(GemmArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[kLds<SIDE>];
  product<PS, QS, SIDE>(a, blockIdx.x, gridDim.x, lds);
}

// Both products of a backward that do not fill the chip one by one, and the sums of the bias's gradient from
// its parts, in one launch.
template <int SIDE>
__global__ __launch_bounds__(256, kPerUnit<SIDE>) void gemm_f32_pair_kernel(GemmPair p) {
  __shared__ __attribute__((aligned(1024))) char lds[kLds<SIDE>];
  const uint32_t id = blockIdx.x;
  if (id < p.wgs_dx) product<false, true, SIDE>(p.dx, id, p.wgs_dx, lds);
  else if (id < p.wgs_dx + p.wgs_dw) product<true, true, SIDE>(p.dw, id - p.wgs_dx, p.wgs_dw, lds);
  else sum_columns<kWaves>(p.sums, id - p.wgs_dx - p.wgs_dw, reinterpret_cast<float(*)[64]>(lds));
}

uint32_t workgroups(const GemmArgs& a, int64_t side) {
  return (uint32_t)(((a.I + side - 1) / side) * ((a.J + side - 1) / side));
}

template <int SIDE>
hipError_t launch(const GemmArgs& a) {
  const dim3 grid(workgroups(a, SIDE) * (uint32_t)a.splits);
  if (a.p_slow) hipLaunchKernelGGL((gemm_f32_kernel<true, true, SIDE>), grid, dim3(256), 0, a.stream, a);
  else if (a.q_slow) hipLaunchKernelGGL((gemm_f32_kernel<false, true, SIDE>), grid, dim3(256), 0, a.stream, a);
  else hipLaunchKernelGGL((gemm_f32_kernel<false, false, SIDE>), grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

template <int SIDE>
hipError_t launch_pair(GemmPair p) {
  p.wgs_dx = workgroups(p.dx, SIDE), p.wgs_dw = workgroups(p.dw, SIDE);
  const uint32_t sums = p.sums.parts ? (uint32_t)((p.sums.cols + 63) / 64) : 0;
  hipLaunchKernelGGL((gemm_f32_pair_kernel<SIDE>), dim3(p.wgs_dx + p.wgs_dw + sums), dim3(256), 0,
                     p.dx.stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_f32(const GemmArgs& a) {
  switch (a.side) {
    case 128: return launch<128>(a);
    case 64: return launch<64>(a);
    default: return launch<32>(a);
  }
}

hipError_t launch_gemm_pair_f32(const GemmPair& p) {
  return p.dx.side == 64 ? launch_pair<64>(p) : launch_pair<32>(p);
}

}  // namespace ringx
