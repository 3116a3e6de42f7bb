// Matrix products of the linear layer in bf16 with fp32 accumulation (gfx950):
//   out[i][j] = sum over r of P(i, r) Q(j, r), then the epilogue of linear.h.
// Forward: P = x, Q = w.  dx: P = dz, Q = w read along its rows.  dw: P = dz, Q = x, both read along
// their rows.
//
// v_mfma_f32_16x16x32_bf16 with Q as its first operand: a lane holds one row i and four neighbouring j at a
// time (32 x 32 x 16, whose accumulators are read and written twice as often, took 4 to 7% more time).  Steps are of
// 64 of r (gemm_feed.h).
//
// Two things bound it.  Power: 8192^3 of normally distributed values, launched again and again, takes the clock from
// 1.9 to 1.4 GHz (it does for the library's product too); zeros take 20% less time.  And what stands beside the
// products: the cores are busy for 73% of the cycles (1390 TFLOP/s; the library's product 87%, 1630), for 62% of them
// at 32768 x 2048 to 6144 with its twelve starts and ends of tiles (75%), with 0.38 LDS instructions to a product
// (0.25); by rocprofv3's counters.  Launches without the barriers took 4% less, deeper buffers (four of 32 of r) 6%
// more, wave tiles of 128 x 128 from four waves as much.

#include "gemm_feed.h"
#include "linear.h"

namespace ringx {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

// Fragments of 16 of the width x 32 of r: lane l has width index l % 16 and r = 8 (l / 16) .. + 7.
template <bool SLOW, int W, int BLOCKS, int BK>
struct Frags {
  using F = Feed<__bf16, SLOW, W, 512>;
  static constexpr int kCols = BLOCKS < 4 ? BLOCKS : 4;   // 64 columns further on the swizzle is the same
  int off[SLOW ? 2 : BK / 32][SLOW ? kCols : 1];
  __device__ __forceinline__ void start(int w0, int lane) {   // w0: the wave's first of the tile
    const int g = lane >> 4;
    if constexpr (!SLOW) {
      const int row = w0 + (lane & 15);
#pragma unroll
      for (int s = 0; s < BK / 32; ++s) off[s][0] = row * (2 * BK) + (((4 * s + g) ^ F::swz(row)) << 4);
    } else {
      const int rr = (lane & 15) >> 2;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < kCols; ++b) {
          const int row = 8 * g + 4 * h + rr;
          const int col = w0 + 16 * b + 4 * (lane & 3);
          off[h][b] = row * (2 * W) + (((col >> 3) ^ F::swz(row)) << 4) + (col & 7) * 2;
        }
    }
  }
  __device__ __forceinline__ bf16x8 get(const char* tile, int s, int b) const {
    if constexpr (!SLOW) {
      return *reinterpret_cast<const bf16x8*>(tile + off[s][0] + b * 16 * 2 * BK);
    } else {
      // blocks 8 further are 256 bytes further, past the swizzle's bits; 4 further turn one of them
      const int o = s * 32 * 2 * W + (b / 8) * 256;
      const int flip = (b / 4 % 2) * 128;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (lds_bf16x4*)(tile + (off[0][b % 4] ^ flip) + o));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (lds_bf16x4*)(tile + (off[1][b % 4] ^ flip) + o));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

constexpr int BK = 64;   // r of a step

// GROUPS = 2: two groups of waves take half of the steps each, for launches that leave a compute unit one tile.
template <int TI, int TJ, int WI, int WJ, int GROUPS>
struct Tile {
  static constexpr int kTI = TI, kTJ = TJ, kWI = WI, kWJ = WJ, kGroups = GROUPS;
  static constexpr int kWaves = WI * WJ, kThreads = 64 * kWaves;   // of a group
  static constexpr int kBI = TI / WI / 16, kBJ = 4;                // 16 x 16 blocks of a wave
  static constexpr int kP = TI * BK * 2, kStage = (TI + TJ) * BK * 2;   // bytes
  static_assert(TJ == WJ * 64 && kBI % (2 * GROUPS) == 0, "waves of 64 columns");
};

// The values of a wave's 16 rows x 64 columns on their way out: x[b][e] is row l % 16, column 16 b + 4 (l / 16)
// + e.  Where rows come in 16-byte pieces, bf16 pairs change places among the four lanes of a row, so that
// each has 16 neighbouring columns: two 16-byte stores, whole 128-byte lines of a row.  Otherwise, through
// LDS, a lane takes one column of row after row.
struct Out {
  static constexpr int kPitch = 65;                 // floats of a staged row
  static constexpr int kStage = 16 * kPitch;        // floats of a wave
  int64_t j0;                                       // the wave's first column
  int n, g;
  bool vec;
  f32x4 bias[4];
  int64_t col[2];                                   // of the lane's two pieces, in an output of heads

  __device__ __forceinline__ void start(const GemmOut& o, int64_t j0_, int lane) {
    j0 = j0_, n = lane & 15, g = lane >> 4;
    vec = o.f32 ? o.J % 4 == 0 : o.J % 8 == 0 && o.d % 8 == 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int64_t j = j0 + 16 * b + 4 * g;
      bias[b] = f32x4{};
      if (o.bias && vec && j < o.J) bias[b] = *reinterpret_cast<const f32x4*>(o.bias + j);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t j = (uint32_t)(j0 + 16 * g + 8 * h);
      col[h] = j;
      if (o.heads) {
        const uint32_t head = j / (uint32_t)o.d;
        col[h] = (int64_t)head * o.tokens * o.d + (j - head * (uint32_t)o.d);
      }
    }
  }
  // register b of lane group g <-> register g of lane group b
  static __device__ __forceinline__ void transpose(u32x2 (&v)[4]) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const auto r = __builtin_amdgcn_permlane32_swap(v[b][w], v[b + 2][w], false, false);
        v[b][w] = r[0], v[b + 2][w] = r[1];
      }
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        const auto r = __builtin_amdgcn_permlane16_swap(v[b][w], v[b + 1][w], false, false);
        v[b][w] = r[0], v[b + 1][w] = r[1];
      }
    }
  }
  // rows' 64 columns in bf16 at p (the row's first value plus the lane's columns), where they exist
  __device__ __forceinline__ void store(__bf16* p, const int64_t (&at)[2], bool live, int64_t J,
                                        const f32x4 (&x)[4]) const {
    u32x2 v[4];
#pragma unroll
    for (int b = 0; b < 4; ++b)
      v[b] = u32x2{pack_bf16x2(x[b][0], x[b][1]), pack_bf16x2(x[b][2], x[b][3])};
    transpose(v);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (live && j0 + 16 * g + 8 * h < J)
        *reinterpret_cast<u32x4*>(p + at[h]) = u32x4{v[2 * h][0], v[2 * h][1], v[2 * h + 1][0], v[2 * h + 1][1]};
  }
  __device__ __forceinline__ void rows(const GemmOut& o, int64_t I, int64_t i0, f32x4 (&x)[4],
                                       float* stage) const {
    const int64_t i = i0 + n;
    const bool live = i < I;
    if (!vec) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) stage[n * kPitch + 16 * b + 4 * g + e] = x[b][e];
      __builtin_amdgcn_wave_barrier();
      const int lane = 16 * g + n;
      const int64_t j = j0 + lane;
      float b1[1] = {o.bias && j < o.J ? o.bias[j] : 0.f};
#pragma unroll 1
      for (int r = 0; r < 16; ++r) {
        float y[1] = {stage[r * kPitch + lane]};
        if (i0 + r < I && j < o.J) finish<1, false, __bf16>(o, i0 + r, j, 1, b1, y);
      }
      __builtin_amdgcn_wave_barrier();
      return;
    }
    const int64_t row = i * o.J;
    if (o.f32) {
      // gradients: no bias, activation or residual
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int64_t j = j0 + 16 * b + 4 * g;
        f32x4* const p = reinterpret_cast<f32x4*>((float*)o.out + row + j);
        if (live && j < o.J) *p = o.accumulate ? *p + x[b] : x[b];
      }
      return;
    }
    const int64_t flat[2] = {j0 + 16 * g, j0 + 16 * g + 8};
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] += bias[b];
    if (o.pre) store((__bf16*)o.pre + row, flat, live, o.J, x);
    if (o.act != RINGX_ACT_NONE) {
      activate_all(x, o.act);
    }
    if (o.residual) {
      u32x2 v[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 y = {};
        if (live && flat[h] < o.J) y = *reinterpret_cast<const u32x4*>((const __bf16*)o.residual + row + flat[h]);
        v[2 * h] = u32x2{y[0], y[1]}, v[2 * h + 1] = u32x2{y[2], y[3]};
      }
      transpose(v);
#pragma unroll
      for (int b = 0; b < 4; ++b)
        x[b] += f32x4{bf16_lo(v[b][0]), bf16_hi(v[b][0]), bf16_lo(v[b][1]), bf16_hi(v[b][1])};
    }
    int64_t first = row;
    if (o.heads) {
      const uint32_t b = (uint32_t)i / (uint32_t)o.tokens, t = (uint32_t)i - b * (uint32_t)o.tokens;
      first = (int64_t)b * o.tokens * o.J + t * o.d;
    }
    store((__bf16*)o.out + first, col, live, o.J, x);
  }
};

// Workgroup `id` of a product.
template <bool PS, bool QS, class C>
__device__ __forceinline__ void product(const GemmArgs& a, const uint32_t id, char* const lds_all) {
  constexpr int TI = C::kTI, TJ = C::kTJ, WJ = C::kWJ, kGroups = C::kGroups;
  static_assert(C::kWaves * Out::kStage * 4 <= 2 * C::kStage, "staging fits");
  const int tid = threadIdx.x % C::kThreads, lane = tid & 63;
  const int wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = kGroups == 1 ? 0 : wave8 / C::kWaves, wave = kGroups == 1 ? wave8 : wave8 % C::kWaves;
  char* const lds = lds_all + group * 2 * C::kStage;
  const uint32_t lbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  // whole tiles first, then the last ones in parts along r
  const uint32_t ti = ((uint32_t)a.I + TI - 1) / TI, tj = ((uint32_t)a.J + TJ - 1) / TJ;
  const uint32_t whole = a.cut.whole, parts = a.cut.parts;
  uint32_t tile, of = 0, i_tile, j_tile;
  const bool split = id >= whole && parts > 1;
  if (id < whole) {
    tile = xcd_remap(id, whole);
  } else {
    tile = whole + (id - whole) / parts;
    of = (id - whole) % parts;
  }
  place(tile, ti, tj, i_tile, j_tile);
  const uint32_t i0 = i_tile * TI, j0 = j_tile * TJ;

  const uint32_t steps = ((uint32_t)a.R + BK - 1) / BK;
  uint32_t s0 = 0, s1 = steps;
  if (split) s0 = steps * of / parts, s1 = steps * (of + 1) / parts;
  // the group's steps; with an odd number of them the second one's last holds zeros
  const int count = (int)(s1 - s0 + kGroups - 1) / kGroups;
  if (kGroups > 1 && group == 0) s1 = s0 + count;
  if (kGroups > 1 && group == 1) s0 = s0 + count;
  Feed<__bf16, PS, TI, C::kThreads> fp;
  Feed<__bf16, QS, TJ, C::kThreads> fq;
  fp.start(a.P, i0, BK * s0, tid);
  fq.start(a.Q, j0, BK * s0, tid);
  const int wi = wave / WJ, wj = wave % WJ;
  Frags<PS, TI, C::kBI, BK> rp;
  Frags<QS, TJ, C::kBJ, BK> rq;
  rp.start(wi * 16 * C::kBI, lane);
  rq.start(wj * 16 * C::kBJ, lane);
  const uint32_t wdst = (uint32_t)__builtin_amdgcn_readfirstlane(lbase + wave * 1024);

  f32x4 acc[C::kBI][C::kBJ];
#pragma unroll
  for (int i = 0; i < C::kBI; ++i)
#pragma unroll
    for (int j = 0; j < C::kBJ; ++j) acc[i][j] = f32x4{};

  // of r, in this part from the step to load on
  int rest = min((int)a.R - (int)(BK * s0), (int)(BK * s1) - (int)(BK * s0));
  // A step is four units: 32 of r, half of the wave's i.  Unit T - 1's products, beside them the reads of unit T
  // of the step in `buf` and L of a later step's loads.
  constexpr int kHalf = C::kBI / 2, kProducts = kHalf * C::kBJ;
  bf16x8 p[2][kHalf], q[2][C::kBJ];
  auto unit = [&](auto t, uint32_t buf, auto feed, auto loads) {
    constexpr int T = decltype(t)::value, L = decltype(loads)::value, U = (T + 3) % 4;
    constexpr int kReadsQ = T % 2 == 0 ? C::kBJ : 0, kFrags = kReadsQ + kHalf;
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
#pragma unroll
      for (int u = i * L / kProducts; u < (i + 1) * L / kProducts; ++u) feed(u);
#pragma unroll
      for (int f = i * kFrags / kProducts; f < (i + 1) * kFrags / kProducts; ++f) {
        if (f < kReadsQ) q[T / 2][f] = rq.get(lds + buf + C::kP, T / 2, f);
        else p[T % 2][f - kReadsQ] = rp.get(lds + buf, T / 2, T % 2 * kHalf + f - kReadsQ);
      }
      f32x4& c = acc[U % 2 * kHalf + i / C::kBJ][i % C::kBJ];
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[U / 2][i % C::kBJ], p[U % 2][i / C::kBJ], c, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto nothing = [](int) {};
  using std::integral_constant;
  typedef integral_constant<int, 0> kNone;
  typedef integral_constant<int, Feed<__bf16, PS, TI, C::kThreads>::kLoads> kLoadsP;
  typedef integral_constant<int, Feed<__bf16, QS, TJ, C::kThreads>::kLoads> kLoadsQ;
  // Two buffers.  A step's buffer is free behind the barrier after its last reads; the loads of two steps
  // later go there, P's beside the products that follow, Q's beside the next ones.  Fragments are read one
  // unit ahead, those of a step's first unit behind that same barrier, so that the last unit's
  // products cover the barrier and the reads.
  fp.all(wdst, rest);
  fq.all(wdst + C::kP, rest);
  rest -= BK;
  fp.all(wdst + C::kStage, rest);
  wait_vmem<kLoadsP::value>();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < C::kBJ; ++j) q[0][j] = rq.get(lds + C::kP, 0, j);
#pragma unroll
  for (int i = 0; i < kHalf; ++i) p[0][i] = rp.get(lds, 0, i);
  uint32_t buf = 0;   // the step's buffer
  for (int s = count; s > 0; --s) {
    fq.begin(rest);
    unit(integral_constant<int, 1>{}, buf,
         [&](int u) { fq.load(u, wdst + C::kStage - buf + C::kP); }, kLoadsQ{});
    rest -= BK;
    unit(integral_constant<int, 2>{}, buf, nothing, kNone{});
    unit(integral_constant<int, 3>{}, buf, nothing, kNone{});
    wait_vmem_all();
    __syncthreads();
    fp.begin(rest);
    buf = C::kStage - buf;
    unit(integral_constant<int, 0>{}, buf, [&](int u) { fp.load(u, wdst + C::kStage - buf); },
         kLoadsP{});
  }
  wait_vmem_all();
  __syncthreads();

  // of the groups' blocks each ends a half, with the other's sums of it through LDS
  constexpr int kOwn = C::kBI / kGroups;
  if constexpr (kGroups == 2) {
    f32x4* const other = reinterpret_cast<f32x4*>(lds_all + (1 - group) * 2 * C::kStage) + tid;
    f32x4* const mine = reinterpret_cast<f32x4*>(lds) + tid;
    static_assert(kOwn * C::kBJ * C::kThreads * 16 <= 2 * C::kStage, "half of the sums fits");
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
#pragma unroll
      for (int b = 0; b < C::kBJ; ++b)
        other[(k * C::kBJ + b) * C::kThreads] = group == 0 ? acc[kOwn + k][b] : acc[k][b];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
#pragma unroll
      for (int b = 0; b < C::kBJ; ++b) {
        const f32x4 x = mine[(k * C::kBJ + b) * C::kThreads];
        if (group == 0) acc[k][b] += x;
        else acc[k][b] = x + acc[kOwn + k][b];
      }
    __syncthreads();
  }
  const int first = group * kOwn;   // acc[0 .. kOwn) are the wave's blocks from here on

  if (split) {
    // as it lies in the registers
    f32x4* const part = reinterpret_cast<f32x4*>(a.part) + (int64_t)(id - whole) * (TI * TJ / 4);
#pragma unroll
    for (int bi = 0; bi < kOwn; ++bi)
#pragma unroll
      for (int bj = 0; bj < C::kBJ; ++bj)
        part[((first + bi) * C::kBJ + bj) * C::kThreads + tid] = acc[bi][bj];
    return;
  }
  Out out;
  out.start(a.o, (int64_t)j0 + wj * 64, lane);
  float* const stage = reinterpret_cast<float*>(lds) + wave * Out::kStage;
  // a loop whose code is there once: unrolled it is 130 KB, which every tile would fetch
#pragma unroll 1
  for (int bi = 0; bi < kOwn; ++bi) {
    f32x4 x[4] = {};
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      if (bi == k) {
        cold_path();
#pragma unroll
        for (int b = 0; b < C::kBJ; ++b) x[b] = acc[k][b];
      }
    }
    out.rows(a.o, a.I, (int64_t)i0 + (wi * C::kBI + first + bi) * 16, x, stage);
  }
}

template <bool PS, bool QS, class C>
__global__ __launch_bounds__(C::kThreads * C::kGroups, 2) void gemm_bf16_kernel(GemmArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[C::kGroups * 2 * C::kStage];
  product<PS, QS, C>(a, blockIdx.x, lds);
}

// The parts of the last tile `rest`, in their order, then the epilogue; bi: which block of 16 rows of every
// wave.
template <class C>
__device__ __forceinline__ void join(const GemmArgs& a, uint32_t rest, int bi, float* lds) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ti = ((uint32_t)a.I + C::kTI - 1) / C::kTI, tj = ((uint32_t)a.J + C::kTJ - 1) / C::kTJ;
  uint32_t i, j;
  place(a.cut.whole + rest, ti, tj, i, j);
  constexpr int64_t kSize = C::kTI * C::kTJ / 4;
  const f32x4* const part =
      reinterpret_cast<const f32x4*>(a.part) + (int64_t)rest * a.cut.parts * kSize + bi * C::kBJ * C::kThreads + tid;
  f32x4 x[4] = {};
#pragma unroll 4
  for (uint32_t s = 0; s < a.cut.parts; ++s)
#pragma unroll
    for (int b = 0; b < C::kBJ; ++b) x[b] += part[s * kSize + b * C::kThreads];
  Out out;
  out.start(a.o, (int64_t)j * C::kTJ + wave % C::kWJ * 64, tid & 63);
  out.rows(a.o, a.I, (int64_t)i * C::kTI + (wave / C::kWJ * C::kBI + bi) * 16, x, lds + wave * Out::kStage);
}

template <class C>
__global__ __launch_bounds__(C::kThreads) void gemm_join_kernel(GemmArgs a) {
  __shared__ float lds[C::kWaves * Out::kStage];
  join<C>(a, blockIdx.x, blockIdx.y, lds);
}

// Both products of a backward that do not fill the chip one by one, and the sums of the bias's gradient from
// its parts, in one launch.
template <class C>
__global__ __launch_bounds__(C::kThreads * C::kGroups, 2) void gemm_pair_kernel(GemmPair p) {
  __shared__ __attribute__((aligned(1024))) char lds[C::kGroups * 2 * C::kStage];
  const uint32_t id = blockIdx.x;
  if (id < p.wgs_dx) {
    product<false, true, C>(p.dx, id, lds);
  } else if (id < p.wgs_dx + p.wgs_dw) {
    product<true, true, C>(p.dw, id - p.wgs_dx, lds);
  } else {
    sum_columns<C::kWaves * C::kGroups>(p.sums, id - p.wgs_dx - p.wgs_dw, reinterpret_cast<float(*)[64]>(lds));
  }
}

template <class C>
__global__ __launch_bounds__(C::kThreads) void gemm_join_pair_kernel(GemmPair p) {
  __shared__ float lds[C::kWaves * Out::kStage];
  if (blockIdx.x < p.rest_dx) join<C>(p.dx, blockIdx.x, blockIdx.y, lds);
  else join<C>(p.dw, blockIdx.x - p.rest_dx, blockIdx.y, lds);
}

// last tiles, those that are cut
uint32_t rest_of(const GemmArgs& a) {
  const int64_t side = a.cut.large ? 256 : 128;
  return (uint32_t)(((a.I + side - 1) / side) * ((a.J + side - 1) / side) - a.cut.whole);
}

template <class C>
hipError_t launch(const GemmArgs& a) {
  const uint32_t rest = rest_of(a);
  const dim3 grid(a.cut.whole + rest * a.cut.parts), threads(C::kThreads * C::kGroups);
  if (a.p_slow) hipLaunchKernelGGL((gemm_bf16_kernel<true, true, C>), grid, threads, 0, a.stream, a);
  else if (a.q_slow) hipLaunchKernelGGL((gemm_bf16_kernel<false, true, C>), grid, threads, 0, a.stream, a);
  else hipLaunchKernelGGL((gemm_bf16_kernel<false, false, C>), grid, threads, 0, a.stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.cut.parts == 1 || rest == 0) return e;
  hipLaunchKernelGGL((gemm_join_kernel<C>), dim3(rest, C::kBI), dim3(C::kThreads), 0, a.stream, a);
  return hipGetLastError();
}

template <class C>
hipError_t launch_pair(GemmPair p) {
  p.rest_dx = rest_of(p.dx), p.rest_dw = rest_of(p.dw);
  p.wgs_dx = p.dx.cut.whole + p.rest_dx * p.dx.cut.parts;
  p.wgs_dw = p.dw.cut.whole + p.rest_dw * p.dw.cut.parts;
  const uint32_t sums = p.sums.parts ? (uint32_t)((p.sums.cols + 63) / 64) : 0;
  hipLaunchKernelGGL((gemm_pair_kernel<C>), dim3(p.wgs_dx + p.wgs_dw + sums),
                     dim3(C::kThreads * C::kGroups), 0, p.dx.stream, p);
  const hipError_t e = hipGetLastError();
  if (p.dx.cut.parts == 1) p.rest_dx = 0;
  if (p.dw.cut.parts == 1) p.rest_dw = 0;
  if (e != hipSuccess || p.rest_dx + p.rest_dw == 0) return e;
  hipLaunchKernelGGL((gemm_join_pair_kernel<C>), dim3(p.rest_dx + p.rest_dw, C::kBI), dim3(C::kThreads), 0,
                     p.dx.stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_bf16(const GemmArgs& a) {
  if (a.cut.large) return launch<Tile<256, 256, 2, 4, 1>>(a);
  if (a.cut.groups == 2) return launch<Tile<128, 128, 2, 2, 2>>(a);
  return launch<Tile<128, 128, 2, 2, 1>>(a);
}

hipError_t launch_gemm_pair_bf16(const GemmPair& p) {
  return p.dx.cut.groups == 2 ? launch_pair<Tile<128, 128, 2, 2, 2>>(p)
                              : launch_pair<Tile<128, 128, 2, 2, 1>>(p);
}

}  // namespace ringx
