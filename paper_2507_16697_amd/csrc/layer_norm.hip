// Layer norm over the last dimension, forward and backward.
//
// Row x of C values: mean = sum x / C, r = (sum (x - mean)^2 / C + eps)^(-1/2), n = (x - mean) r,
// y = n w + b.  Backward, g = dy w:
//   dx = r (g - sum g / C - n sum(g n) / C) (+ dres),   dw = sum over rows of dy n,   db = sum of dy.
//
// Bound by HBM: x is read and y written once, backward x, dy and dres are read and dx written once.  A row
// is held in registers by TPR threads, E values each, from its load to its store, so that the squares
// are those of the differences from the mean (a second sum of the differences takes back the rounding of
// the first mean).  Threads keep their columns for all rows that they take: weights are loaded once, and
// the weights' gradients add up in registers until the workgroup writes one row of parts at its end.

#include "ringx_device.h"
#include "ringx_kernels.h"

#include <algorithm>
#include <type_traits>

namespace ringx {
namespace {

// The E values of a row that one thread holds: pieces of V values (16 bytes; 4 of bf16; one), piece v at columns
// (v TPR + t) V.  Columns past C are zero.  (bf16 in pieces of 4 bytes against one by one: 32768 x 2046 backward 85
// us, 109; 8192 x 5002 forward 42, 67.)
template <class T, int V_, int E, int TPR>
struct Row {
  static constexpr int V = V_;
  static_assert(V == 1 || V * sizeof(T) == 16 || V * sizeof(T) == 4, "pieces");
  static constexpr int NV = E / V;
  static constexpr int kPiece = V * (int)sizeof(T) / 4, kWords = V > 1 ? NV * kPiece : E;   // words
  uint32_t w[kWords];

  static __device__ __forceinline__ int col(int e, int t) { return (e / V * TPR + t) * V + e % V; }

  __device__ __forceinline__ void load(const T* p, int t, int C) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = col(v * V, t);
      if constexpr (kPiece == 4) {
        u32x4 x = {};
        if (c < C) x = *reinterpret_cast<const u32x4*>(p + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * v + j] = x[j];
      } else if constexpr (V > 1) {
        w[v] = 0u;
        if (c < C) w[v] = *reinterpret_cast<const uint32_t*>(p + c);
      } else {
        w[v] = 0u;
        if (c < C) w[v] = raw_bits(p + c);
      }
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (V == 1 || std::is_same_v<T, float>) return from_raw<T>(w[e]);
    else return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
  }
  // Small pieces, each loaded under its condition, have arrived: nothing that uses them joins their
  // conditional blocks, where it would wait for every load alone (bf16, 4000 rows of 2047, backward: 121 -> 31 us;
  // fp32's use joins none).
  __device__ __forceinline__ void arrived() {
    if constexpr (kPiece < 4 && std::is_same_v<T, __bf16>) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
  }
  static __device__ __forceinline__ void store(T* p, int t, int C, const float (&x)[E]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = col(v * V, t);
      if (c >= C) continue;
      if constexpr (kPiece == 4) {
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (std::is_same_v<T, float>) y[j] = __float_as_uint(x[v * V + j]);
          else y[j] = pack_bf16x2(x[v * V + 2 * j], x[v * V + 2 * j + 1]);
        }
        *reinterpret_cast<u32x4*>(p + c) = y;
      } else if constexpr (V > 1) {
        *reinterpret_cast<uint32_t*>(p + c) = pack_bf16x2(x[v * V], x[v * V + 1]);
      } else {
        p[c] = (T)x[v];
      }
    }
  }
};

// fp32 values of the thread's columns, min(V, 4) at a time
template <class R>
constexpr int kAtOnce = R::V < 4 ? R::V : 4;
template <class R, int E>
__device__ __forceinline__ void load_floats(const float* p, float otherwise, int t, int C, float (&x)[E]) {
  constexpr int N = kAtOnce<R>;
  typedef __attribute__((ext_vector_type(N))) float Piece;
#pragma unroll
  for (int e = 0; e < E; e += N) {
    const int c = R::col(e, t);
    Piece y = otherwise;
    if (p && c < C) y = *reinterpret_cast<const Piece*>(p + c);
#pragma unroll
    for (int j = 0; j < N; ++j) x[e + j] = y[j];
  }
}
template <class R, int E>
__device__ __forceinline__ void store_floats(float* p, int t, int C, const float (&x)[E]) {
  constexpr int N = kAtOnce<R>;
  typedef __attribute__((ext_vector_type(N))) float Piece;
  if (!p) return;
#pragma unroll
  for (int e = 0; e < E; e += N) {
    const int c = R::col(e, t);
    if (c >= C) continue;
    Piece y;
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = x[e + j];
    *reinterpret_cast<Piece*>(p + c) = y;
  }
}

// The same columns of a row of G, fp32 beside a bf16 x.
template <class T, class G, int V, int E, int TPR>
struct GradRow : Row<T, V, E, TPR> {};
template <int V, int E, int TPR>
struct GradRow<__bf16, float, V, E, TPR> {
  float w[E];
  __device__ __forceinline__ void load(const float* p, int t, int C) {
    load_floats<Row<__bf16, V, E, TPR>>(p, 0.f, t, C, w);
  }
  __device__ __forceinline__ float get(int e) const { return w[e]; }
  __device__ __forceinline__ void arrived() {
    if constexpr (V < 8) {
#pragma unroll
      for (int e = 0; e < E; ++e) asm volatile("" : "+v"(w[e]));
    }
  }
};

template <int CTRL>
__device__ __forceinline__ float add_lane(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ float lane_sum(float x) {   // over N <= 64 neighbouring lanes, in each
  if constexpr (N >= 2) x = add_lane<0xB1>(x);     // lanes 1 0 3 2 of every four
  if constexpr (N >= 4) x = add_lane<0x4E>(x);     // lanes 2 3 0 1
  if constexpr (N >= 8) x = add_lane<0x141>(x);    // mirrored in eight: the other four
  if constexpr (N >= 16) x = add_lane<0x140>(x);   // mirrored in sixteen: the other eight
  if constexpr (N >= 32) x += __shfl_xor(x, 16, 64);
  if constexpr (N >= 64) x = sum_halves(x);
  return x;
}

// Threads of a workgroup.  Rows of up to 64 threads share 256.  Wider ones have one of their own forward (8192 x
// 8192 bf16 44 us, sharing 512 56) and share 512 backward, where a workgroup has parts to write (99 -> 91 us with half
// as many of them).
template <int TPR, bool BWD>
constexpr int kGroup = TPR <= 64 ? 256 : BWD && TPR <= 512 ? 512 : TPR;
template <int TPR, bool BWD>
constexpr int kRowsAtOnce = kGroup<TPR, BWD> / TPR;

// Sums of two values over the TPR threads of a row.  Rows of several waves go through LDS, `slot`
// alternating, so that one barrier serves: a slot is written again two sums later, behind the next one's
// barrier.  Lanes and waves are added up as trees: with a thread's own values, 32 of them at most, a sum of a row is
// off by at most 41 half steps of its terms' sizes.  Up to eight waves a thread adds up itself, sixteen it adds
// over lanes (4096 x 12002 bf16 forward 56 us, with eight over lanes 58; registers for sixteen would spill).
constexpr int log2_of(int n) { return n > 1 ? 1 + log2_of(n / 2) : 0; }
template <int TPR, int E>
constexpr int kRowSteps = E + log2_of(TPR);

template <int TPR, bool BWD>
struct RowSum {
  f32x2 lds[2][kGroup<TPR, BWD> / 64];
  __device__ __forceinline__ f32x2 operator()(float a, float b, int& slot) {
    a = lane_sum<(TPR < 64 ? TPR : 64)>(a);
    b = lane_sum<(TPR < 64 ? TPR : 64)>(b);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0) lds[slot][threadIdx.x >> 6] = f32x2{a, b};
      __syncthreads();
      constexpr int kWaves = TPR / 64;
      const f32x2* const x = lds[slot] + threadIdx.x / TPR * kWaves;
      if constexpr (kWaves <= 8) {
        f32x2 y[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) y[i] = x[i];
#pragma unroll
        for (int n = 1; n < kWaves; n *= 2)
#pragma unroll
          for (int i = 0; i < kWaves; i += 2 * n) y[i] += y[i + n];
        a = y[0][0], b = y[0][1];
      } else {
        const f32x2 y = x[threadIdx.x % kWaves];
        a = lane_sum<kWaves>(y[0]), b = lane_sum<kWaves>(y[1]);
      }
      slot ^= 1;
    }
    return f32x2{a, b};
  }
};

template <class T, int V, int E, int TPR>
__global__ __launch_bounds__((kGroup<TPR, false>)) void layer_norm_kernel(NormArgs a) {
  static_assert(kRowSteps<TPR, E> <= 41, "the bound of a row's sums");
  using R = Row<T, V, E, TPR>;
  __shared__ RowSum<TPR, false> sum;
  const int t = threadIdx.x % TPR;
  const int C = a.C;
  const float inv = 1.f / (float)C;
  const int64_t step = (int64_t)gridDim.x * kRowsAtOnce<TPR, false>;
  int64_t row = (int64_t)blockIdx.x * kRowsAtOnce<TPR, false> + threadIdx.x / TPR;
  const T* const x = (const T*)a.x;
  T* const y = (T*)a.y;
  R cur;
  // rows past the end (of the last round) repeat the last one and are not stored
  cur.load(x + min(row, a.rows - 1) * a.stride, t, C);
  float w[E], b[E];
  load_floats<R>(a.weight, 1.f, t, C, w);
  load_floats<R>(a.bias, 0.f, t, C, b);
  int slot = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * kRowsAtOnce<TPR, false>; r0 < a.rows; r0 += step, row += step) {
    R next;
    if (r0 + step < a.rows) next.load(x + min(row + step, a.rows - 1) * a.stride, t, C);
    float s = 0.f, d[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s += cur.get(e);
    float m0 = sum(s, 0.f, slot)[0] * inv;
    asm("" : "+v"(m0));   // rounded here once: the differences and the mean below are from the same m0
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      d[e] = R::col(e, t) < C ? cur.get(e) - m0 : 0.f;
      s1 += d[e];
      s2 = __builtin_fmaf(d[e], d[e], s2);
    }
    const f32x2 ss = sum(s1, s2, slot);
    const float m1 = ss[0] * inv;   // what m0 is off by
    const float var = __builtin_fmaf(-m1, m1, ss[1] * inv);
    const float r = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);   // a row that holds NaN has none
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = __builtin_fmaf((d[e] - m1) * r, w[e], b[e]);
    if (row < a.rows) {
      R::store(y + row * C, t, C, d);
      if (a.stats && t == 0) a.stats[row] = m0 + m1, a.stats[a.rows + row] = r;
    }
    cur = next;
  }
}

template <class T, class G, int V, int E, int TPR>
__global__ __launch_bounds__((kGroup<TPR, true>), TPR <= 256 ? 2 : 1) void layer_norm_bwd_kernel(NormArgs a) {
  static_assert(kRowSteps<TPR, E> <= 41, "the bound of a row's sums");
  using R = Row<T, V, E, TPR>;
  __shared__ RowSum<TPR, true> sum;
  constexpr int kPitch = TPR + 1;   // of a thread's e-th values in LDS: neither way meets itself in a bank
  __shared__ float lds[kRowsAtOnce<TPR, true> > 1 ? 2 * E * kPitch : 1];
  const int t = threadIdx.x % TPR;
  const int C = a.C;
  const float inv = 1.f / (float)C;
  const int64_t step = (int64_t)gridDim.x * kRowsAtOnce<TPR, true>;
  const T *const x = (const T*)a.x, *const dres = (const T*)a.dres;
  const G* const dy = (const G*)a.dy;
  T* const dx = (T*)a.dx;
  float w[E], dw[E], db[E];
  load_floats<R>(a.weight, 1.f, t, C, w);
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
  int slot = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * kRowsAtOnce<TPR, true>; r0 < a.rows; r0 += step) {
    const int64_t at = r0 + threadIdx.x / TPR;
    const bool live = at < a.rows;
    const int64_t row = live ? at : a.rows - 1;   // rows past the end repeat the last one
    R rx, rr;
    GradRow<T, G, V, E, TPR> rg;
    rx.load(x + row * a.stride, t, C);
    rg.load(dy + row * C, t, C);
    if (dres) rr.load(dres + row * C, t, C);
    const float mean = a.stats_in[row], r = a.stats_in[a.rows + row];
    rx.arrived();
    rg.arrived();
    float n[E], g[E], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      n[e] = R::col(e, t) < C ? (rx.get(e) - mean) * r : 0.f;
      g[e] = rg.get(e) * w[e];
      s1 += g[e];
      s2 = __builtin_fmaf(g[e], n[e], s2);
      if (live) {
        dw[e] = __builtin_fmaf(rg.get(e), n[e], dw[e]);
        db[e] += rg.get(e);
      }
    }
    const f32x2 ss = sum(s1, s2, slot);
    const float m1 = ss[0] * inv, m2 = ss[1] * inv;
    if (dres) rr.arrived();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      g[e] = r * (g[e] - m1 - n[e] * m2);
      if (dres) g[e] += rr.get(e);
    }
    if (live) R::store(dx + row * C, t, C, g);
  }
  if (!a.part) return;
  // the workgroup's parts; a launch of one has the sums
  const bool alone = gridDim.x == 1;
  float* const part = a.part + (int64_t)blockIdx.x * 2 * C;
  float* const pw = alone ? a.dweight : part;
  float* const pb = alone ? a.dbias : part + C;
  if constexpr (kRowsAtOnce<TPR, true> == 1) {
    store_floats<R>(pw, t, C, dw);
    store_floats<R>(pb, t, C, db);
  } else {
    // over the rows of a wave, then row after row (of waves)
    constexpr int kHeld = TPR < 64 ? 64 : TPR;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int off = TPR; off < 64; off <<= 1) {
        dw[e] += __shfl_xor(dw[e], off, 64);
        db[e] += __shfl_xor(db[e], off, 64);
      }
    float *const sw = lds + t, *const sb = sw + E * kPitch;
    for (int i = 0; i < kGroup<TPR, true> / kHeld; ++i) {
      if ((int)threadIdx.x / kHeld == i && threadIdx.x % kHeld < TPR) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sw[e * kPitch] = dw[e] + (i ? sw[e * kPitch] : 0.f);
          sb[e * kPitch] = db[e] + (i ? sb[e * kPitch] : 0.f);
        }
      }
      __syncthreads();
    }
    // neighbouring columns in neighbouring lanes: 4 bytes to a lane 32 apart took 20 us of 95 at 8192 x 8192 bf16
    for (int c = threadIdx.x; c < C; c += kGroup<TPR, true>) {
      const int at = (c / (R::V * TPR) * R::V + c % R::V) * kPitch + c / R::V % TPR;
      if (pw) pw[c] = lds[at];
      if (pb) pb[c] = lds[E * kPitch + at];
    }
  }
}

template <class T, class G, int V, int E, int TPR>
hipError_t launch_as(const NormArgs& a, bool bwd) {
  const int64_t at_once = bwd ? kRowsAtOnce<TPR, true> : kRowsAtOnce<TPR, false>;
  const int64_t groups = (a.rows + at_once - 1) / at_once;
  int64_t grid = std::min<int64_t>(groups, norm_workgroups(a.C, bwd));
  // Few rows: one workgroup, four rounds at most (5 us), and no second launch (4 us, and as much of the host).
  if (bwd && a.part && groups <= 4) grid = 1;
  if (!bwd) {
    hipLaunchKernelGGL((layer_norm_kernel<T, V, E, TPR>), dim3((uint32_t)grid), dim3(kGroup<TPR, false>), 0,
                       a.stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((layer_norm_bwd_kernel<T, G, V, E, TPR>), dim3((uint32_t)grid), dim3(kGroup<TPR, true>), 0,
                     a.stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part || grid == 1) return e;
  ColumnSums s;
  s.part = a.part, s.parts = (int)grid, s.cols = 2 * a.C, s.split = a.C;
  s.out[0] = a.dweight, s.out[1] = a.dbias, s.stream = a.stream;
  return launch_column_sums(s);
}

template <class T, int V, int E, int TPR>
hipError_t launch(const NormArgs& a, bool bwd) {
  if (bwd && a.dy_f32) return launch_as<T, float, V, E, TPR>(a, bwd);
  return launch_as<T, T, V, E, TPR>(a, bwd);
}

template <class T, int V>
hipError_t by_width(const NormArgs& a, bool bwd) {
  if (a.C <= 64) return launch<T, V, 8, 8>(a, bwd);
  if (a.C <= 128) return launch<T, V, 8, 16>(a, bwd);
  if (a.C <= 256) return launch<T, V, 8, 32>(a, bwd);
  if (a.C <= 512) return launch<T, V, 8, 64>(a, bwd);
  if (a.C <= 1024) return launch<T, V, 16, 64>(a, bwd);
  // 32 values to a thread in 16-byte pieces of bf16, and past 8192 columns also in pairs (4096 x 12002 backward 82 us,
  // with 16 118; 16384 x 3002 forward 45, 40).  The others' backward would not keep them in registers; with 16, only
  // the widest rows' does not, of 1024 threads.
  constexpr int E = V == 8 ? 32 : 16, W = V > 1 && std::is_same_v<T, __bf16> ? 32 : 16;
  if (a.C <= 2048) return launch<T, V, E, 2048 / E>(a, bwd);
  if (a.C <= 4096) return launch<T, V, E, 4096 / E>(a, bwd);
  if (a.C <= 8192) return launch<T, V, E, 8192 / E>(a, bwd);
  return launch<T, V, W, 16384 / W>(a, bwd);
}

}  // namespace

hipError_t launch_layer_norm(const NormArgs& a, bool bwd) {
  if (!a.bf16) return a.piece == 4 ? by_width<float, 4>(a, bwd) : by_width<float, 1>(a, bwd);
  if (a.piece == 8) return by_width<__bf16, 8>(a, bwd);
  return a.piece == 2 ? by_width<__bf16, 2>(a, bwd) : by_width<__bf16, 1>(a, bwd);
}

}  // namespace ringx
