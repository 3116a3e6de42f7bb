// Matrix products of the linear layer in bf16 with fp32 accumulation (gfx950):
//   out[i][j] = sum over r of P(i, r) Q(j, r), then the epilogue of linear.h.
// Forward: P = x, Q = w.  dx: P = dz, Q = w read along its rows.  dw: P = dz, Q = x, both read along
// their rows.
//
// A workgroup makes a TI x TJ tile of out.  Operands go through LDS in steps of 64 along r, two buffers
// filled by direct global->LDS loads: while one step is multiplied, the next one is in flight.  An operand
// that is stored with r along its rows (contiguous) is a tile of W rows x 64; one stored the other way
// (slow: r is the row) a tile of 64 rows x W, whose fragments come from transposed LDS reads.  16-byte
// pieces of a row are XOR-swizzled by the row so that neither kind of read meets itself in a bank:
// contiguous tiles, 128 bytes a row, by (row / 2) mod 8 (16 lanes read one piece of 16 rows); slow tiles by
// 4 (row mod 4) + (row / 4) mod 4 (16 lanes read 32 bytes of 4 rows).
//
// All loads are buffer loads from the tile's place on: what lies past the tensor's end reads as zero, and
// so do the pieces past R in the last step, whose offsets are moved outside.  Rows of i or j past the
// end repeat the last one (contiguous) or are what follows (slow): they reach only values that are not
// stored.
//
// v_mfma_f32_32x32x16_bf16 with Q as its first operand: a lane holds one row i and four neighbouring j at a
// time.  The waves pass their values through LDS, 32 rows of i at a time, so that the epilogue has 8
// neighbouring j of one row in a lane: 16-byte loads and stores, 128 bytes of a row in a piece.

#include "linear.h"

#ifndef V_WJ
#define V_WJ 4
#endif
#ifndef V_BK
#define V_BK 64
#endif
#ifndef V_NS
#define V_NS 2
#endif
#ifndef V_BK2
#define V_BK2 64
#endif
#ifndef V_NS2
#define V_NS2 2
#endif
namespace ringx {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr uint32_t kOutside = 0x80000000u;   // a byte offset past any buffer here
constexpr uint32_t kMostBytes = 0x7ffffff0u;

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// One 16-byte direct buffer->LDS load per lane; LDS destination lds_base + 16 lane.  Volatile asm for the
// same reasons as the global form in ringx_device.h.
__device__ __forceinline__ void buffer_lds16(const u32x4& rsrc, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds_base), "v"(off), "s"(rsrc)
               : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return reinterpret_cast<int64_t>(uniform_ptr(reinterpret_cast<const void*>(x)));
}

// One operand's way into LDS, BK of r at a time.
template <bool SLOW, int W, int THREADS, int BK>
struct Feed {
  static constexpr int kLoads = W * BK * 2 / (THREADS * 16);
  static constexpr int kRowChunks = SLOW ? W / 8 : BK / 8;
  static_assert(kLoads * THREADS * 16 == W * BK * 2 && (!SLOW || W >= 128), "whole rounds of loads");
  static_assert(SLOW || THREADS / kRowChunks % 16 == 0, "rounds keep the swizzle's phase");
  uint32_t off[kLoads];
  int64_t base, left;    // address of the step's first row or column; bytes from it to the tensor's end
  int64_t step, turn;    // bytes to the next step; what is added where a head (or batch) ends
  int in, per;           // steps left in this head (or batch), steps of one (0: there are none)
  int chunk;             // contiguous: the lane's first r of a step / 8

  static __device__ __forceinline__ int swz(int row) {
    if (SLOW) return ((row & 3) << 2) | ((row >> 2) & 3);
    return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
  }

  // width index w0 and r0 (a multiple of BK) on
  __device__ __forceinline__ void start(const GemmIn& x, int64_t w0, int64_t r0, int tid) {
    const int64_t total = x.heads ? x.rows * x.cols : (x.rows - 1) * x.ld + x.cols;
    int64_t at;   // elements from the tensor's start
    turn = 0, per = 0, in = 0;
    if constexpr (!SLOW) {
      if (x.heads) {
        const int64_t b = w0 / x.tokens;
        const int hd = (int)(x.d / BK), s = (int)(r0 / BK);
        at = b * x.tokens * x.cols + s / hd * x.tokens * x.d + s % hd * BK;
        step = 2 * BK, per = hd, in = hd - s % hd;
        turn = (x.tokens * x.d - x.d) * 2;
      } else {
        at = w0 * x.ld + r0;
        step = 2 * BK;
      }
    } else if (x.heads) {
      const int64_t b = r0 / x.tokens, t = r0 % x.tokens;
      at = b * x.tokens * x.cols + t * x.d;
      step = 2 * BK * x.d, per = (int)(x.tokens / BK), in = (int)((x.tokens - t) / BK);
      turn = (x.cols - x.d) * x.tokens * 2;
    } else {
      at = r0 * x.ld + w0;
      step = 2 * BK * x.ld;
    }
    base = uniform64(reinterpret_cast<int64_t>(x.p) + 2 * at);
    left = uniform64(2 * (total - at));
    chunk = 0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int slot = u * THREADS + tid;
      const int row = slot / kRowChunks;
      const int c = (slot % kRowChunks) ^ swz(row);
      if constexpr (!SLOW) {
        chunk = c;   // the same for every u: rounds are whole multiples of 16 rows
        const int64_t i = min(w0 + row, x.rows - 1);
        int64_t o = (i - w0) * x.ld;
        if (x.heads) {
          const uint32_t b0 = (uint32_t)w0 / (uint32_t)x.tokens, b = (uint32_t)i / (uint32_t)x.tokens;
          o = (int64_t)(b - b0) * x.tokens * x.cols + (i - (int64_t)b * x.tokens) * x.d;
        }
        off[u] = (uint32_t)(2 * o) + c * 16;
      } else {
        int64_t o = row * x.ld + c * 8;
        if (x.heads) {
          const uint32_t col = (uint32_t)min(w0 + c * 8, x.cols - 8);
          const uint32_t h = col / (uint32_t)x.d;
          o = h * x.tokens * x.d + (col - h * (uint32_t)x.d) + row * x.d;
        }
        off[u] = (uint32_t)(2 * o);
      }
    }
  }
  // The loads of a step whose first r has `rest` of them left (none: nothing is read, zeros arrive), one
  // by one, then on to the next step.  No branch, so that a loop's body stays one.
  u32x4 rsrc;
  bool inside;
  __device__ __forceinline__ void begin(int rest) {
    const uint32_t n = left <= 0 ? 0u : left > (int64_t)kMostBytes ? kMostBytes : (uint32_t)left;
    rsrc = u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, rest > 0 ? n : 0u, 0x00020000u};
    inside = SLOW || chunk * 8 < rest;
    int64_t s = step;
    --in;
    const bool end = per && in == 0;
    s += end ? turn : 0, in = end ? per : in;
    base += s, left -= s;
  }
  __device__ __forceinline__ void load(int u, uint32_t dst) const {   // dst: the wave's place
    buffer_lds16(rsrc, inside ? off[u] : kOutside, dst + u * THREADS * 16);
  }
  __device__ __forceinline__ void all(uint32_t dst, int rest) {
    begin(rest);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) load(u, dst);
  }
};

// Fragments of 16 of the width x 32 of r: lane l has width index l % 16 and r = 8 (l / 16) .. + 7.
template <bool SLOW, int W, int BLOCKS, int BK>
struct Frags {
  using F = Feed<SLOW, W, 512, BK>;
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

template <int TI, int TJ, int WI, int WJ, int BK, int NS>
struct Tile {
  static constexpr int kThreads = 64 * WI * WJ;
  static constexpr int kBI = TI / WI / 16, kBJ = TJ / WJ / 16;   // 16 x 16 blocks of a wave
  static constexpr int kP = TI * BK * 2, kStage = (TI + TJ) * BK * 2;   // bytes
  static constexpr int kPitch = 16 * kBJ + 4;                     // floats of a staged row
  static_assert(BK == 64 && WI * WJ * 32 * kPitch * 4 <= NS * kStage, "staging fits");
};

template <bool PS, bool QS, int TI, int TJ, int WI, int WJ, int BK, int NS>
__global__ __launch_bounds__(64 * WI * WJ, TI * TJ > 64 * 128 * WI * WJ ? 1 : 2) void gemm_bf16_kernel(
    GemmArgs a) {
  using C = Tile<TI, TJ, WI, WJ, BK, NS>;
  __shared__ __attribute__((aligned(1024))) char lds[NS * C::kStage];
  const uint32_t lbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // the workgroup's tile: tiles in groups of 4 along i, so that those at work on one XCD share operands
  constexpr uint32_t kGroup = 4;
  const uint32_t ti = (uint32_t)((a.I + TI - 1) / TI), tj = (uint32_t)((a.J + TJ - 1) / TJ);
  uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t split = id / (ti * tj);
  id -= split * ti * tj;
  const uint32_t g0 = id / (kGroup * tj) * kGroup, gn = min(kGroup, ti - g0);
  id -= g0 * tj;
  const int64_t i0 = (int64_t)(g0 + id % gn) * TI, j0 = (int64_t)(id / gn) * TJ;

  const int64_t steps = (a.R + BK - 1) / BK;
  const int64_t s0 = steps * split / a.splits, s1 = steps * (split + 1) / a.splits;
  Feed<PS, TI, C::kThreads, BK> fp;
  Feed<QS, TJ, C::kThreads, BK> fq;
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

  int rest = (int)min(a.R - BK * s0, BK * (s1 - s0));   // of r, in this part from the step to load on
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
  typedef integral_constant<int, Feed<PS, TI, C::kThreads, BK>::kLoads> kLoadsP;
  typedef integral_constant<int, Feed<QS, TJ, C::kThreads, BK>::kLoads> kLoadsQ;
  constexpr int kLoads = kLoadsP::value + kLoadsQ::value;
  auto after = [](uint32_t buf) { return buf == (NS - 1) * C::kStage ? 0u : buf + C::kStage; };
  // NS buffers.  A step's buffer is free behind the barrier after its last reads; the loads of NS steps
  // later go there, P's beside the products that follow, Q's beside the next ones.  Fragments are read one
  // part ahead, those of a step's first part behind that same barrier, so that the last part's
  // products cover the barrier and the reads.
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    fp.all(wdst + n * C::kStage, rest);
    if (n < NS - 1) {
      fq.all(wdst + n * C::kStage + C::kP, rest);
      rest -= BK;
    }
  }
  wait_vmem<(NS - 2) * kLoads + kLoadsP::value>();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < C::kBJ; ++j) q[0][j] = rq.get(lds + C::kP, 0, j);
#pragma unroll
  for (int i = 0; i < kHalf; ++i) p[0][i] = rp.get(lds, 0, i);
  uint32_t buf = 0, last = (NS - 1) * C::kStage;   // the step's buffer, that of the step before it
  for (int s = (int)(s1 - s0); s > 0; --s) {
    fq.begin(rest);
    unit(integral_constant<int, 1>{}, buf, [&](int u) { fq.load(u, wdst + last + C::kP); }, kLoadsQ{});
    rest -= BK;
    unit(integral_constant<int, 2>{}, buf, nothing, kNone{});
    unit(integral_constant<int, 3>{}, buf, nothing, kNone{});
    wait_vmem<(NS - 2) * kLoads>();
    __syncthreads();
    fp.begin(rest);
    last = buf, buf = after(buf);
    unit(integral_constant<int, 0>{}, buf, [&](int u) { fp.load(u, wdst + last); }, kLoadsP{});
  }
  wait_vmem_all();
  __syncthreads();

  // epilogue, 32 rows of i at a time, in the wave's own part of LDS
  GemmOut o = a.o;
  float* const stage = reinterpret_cast<float*>(lds) + wave * 32 * C::kPitch;
  constexpr int kPer = 2 * C::kBJ, kRows = 64 / kPer;   // lanes of a row, rows at a time
  const int jc = lane % kPer * 8;
  const int64_t j = j0 + wj * 16 * C::kBJ + jc;
  const int inside = (int)max((int64_t)0, min((int64_t)8, a.J - j));
  const bool vec = a.J % 8 == 0 && o.d % 8 == 0;
  if (a.splits > 1) {
    o = GemmOut{};
    o.out = a.part + split * a.I * a.J, o.J = a.J, o.f32 = true;
  }
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = o.bias && e < inside ? o.bias[j + e] : 0.f;
#pragma unroll
  for (int bi = 0; bi < C::kBI; bi += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int bj = 0; bj < C::kBJ; ++bj)
        *reinterpret_cast<f32x4*>(stage + (16 * h + (lane & 15)) * C::kPitch + 16 * bj + 4 * (lane >> 4)) =
            acc[bi + h][bj];
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int it = 0; it < 32 / kRows; ++it) {
      const int row = it * kRows + lane / kPer;
      const int64_t i = i0 + (wi * C::kBI + bi) * 16 + row;
      const float* const at = stage + row * C::kPitch + jc;
      if (i >= a.I) continue;
      if (vec) {
        if (inside == 0) continue;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
        float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        finish<8, true, __bf16>(o, i, j, 8, bias, x);
      } else {
#pragma unroll 1
        for (int e = 0; e < inside; ++e) {
          float b1[1] = {o.bias ? o.bias[j + e] : 0.f}, x[1] = {at[e]};
          finish<1, false, __bf16>(o, i, j + e, 1, b1, x);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <bool PS, bool QS, int TI, int TJ, int WI, int WJ, int BK, int NS>
hipError_t launch(const GemmArgs& a) {
  const int64_t tiles = ((a.I + TI - 1) / TI) * ((a.J + TJ - 1) / TJ) * a.splits;
  hipLaunchKernelGGL((gemm_bf16_kernel<PS, QS, TI, TJ, WI, WJ, BK, NS>), dim3((uint32_t)tiles),
                     dim3(64 * WI * WJ), 0, a.stream, a);
  return hipGetLastError();
}

template <int TI, int TJ, int WI, int WJ, int BK, int NS>
hipError_t by_layout(const GemmArgs& a) {
  if (a.p_slow) return launch<true, true, TI, TJ, WI, WJ, BK, NS>(a);
  return a.q_slow ? launch<false, true, TI, TJ, WI, WJ, BK, NS>(a)
                  : launch<false, false, TI, TJ, WI, WJ, BK, NS>(a);
}

}  // namespace

hipError_t launch_gemm_bf16(const GemmArgs& a) {
  return gemm_bf16_large(a.I, a.J) ? by_layout<256, 256, 2, V_WJ, V_BK, V_NS>(a) : by_layout<128, 128, 2, 2, V_BK2, V_NS2>(a);
}

}  // namespace ringx
