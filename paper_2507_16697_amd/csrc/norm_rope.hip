// From a packed projection to the attention's operands, and back: RMS norm of every query and key
// head, rotation by position, and the change from token-major to [B, H, N, d], in one pass.
//
// Row x (one token, one head, d dims), r = (mean x^2 + eps)^(-1/2), y_i = x_i r w_i (w = 1 without
// weights).  The rotated dims are consecutive sections, one per axis of the position; section a of
// 2 n dims from dim o turns its pairs (y_{o+i}, y_{o+n+i}), i < n, by the angle pos_a f_{a,i}:
//   q_{o+i} = y_{o+i} cos - y_{o+n+i} sin,   q_{o+n+i} = y_{o+n+i} cos + y_{o+i} sin.
// Dims after the sections and all of v pass as they are.  Backward, with g the gradient turned back
// (the same with -sin):  dw_i = sum g_i x_i r,  dx_i = r (g_i w_i - x_i r mean_j(g_j w_j x_j r)).
//
// Bound by HBM: every row is read and written once.  A row is held by d / 8 lanes (bf16) or d / 4
// rounded up to a power of two (fp32), 16 bytes each, and a lane keeps its dims for all heads of
// its token: so the sines and cosines, one per held dim, are formed once per token, the weights
// once per wave, and the gradients of the weights add up in registers.  The other member of a pair
// may lie in any lane of the row and comes through LDS.
//
// Angles are formed in 64 bits, as a fraction of a turn: in 32 bits a position of 5e5 would leave
// 0.03 of a radian.

#include "ringx_device.h"
#include "ringx_kernels.h"

#include <algorithm>
#include <type_traits>

namespace ringx {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBatch = 4;   // rows of a lane in flight

// Dims per lane: 16 bytes of the storage type.
template <class T>
constexpr int kHeld = std::is_same_v<T, float> ? 4 : 8;

// kHeld dims of a row from p; VEC: 16-byte accesses, else one by one where dim < d.
template <class T, bool VEC>
__device__ __forceinline__ void load_row(const T* p, int dim, int d, float (&x)[kHeld<T>]) {
  if constexpr (VEC) {
    if (dim < d) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p + dim);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (std::is_same_v<T, float>) {
          x[j] = __uint_as_float(w[j]);
        } else {
          x[2 * j] = bf16_lo(w[j]);
          x[2 * j + 1] = bf16_hi(w[j]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kHeld<T>; ++j) x[j] = 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kHeld<T>; ++j) x[j] = dim + j < d ? (float)p[dim + j] : 0.f;
  }
}
template <class T, bool VEC>
__device__ __forceinline__ void store_row(T* p, int dim, int d, const float (&x)[kHeld<T>]) {
  if constexpr (VEC) {
    if (dim >= d) return;
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same_v<T, float>) w[j] = __float_as_uint(x[j]);
      else w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
    }
    *reinterpret_cast<u32x4*>(p + dim) = w;
  } else {
#pragma unroll
    for (int j = 0; j < kHeld<T>; ++j)
      if (dim + j < d) p[dim + j] = (T)x[j];
  }
}

// What a lane knows of its dims: for each the partner's place in the wave's LDS block and the angle's
// frequency (turns per position) and axis; unrotated dims have frequency 0 and themselves for partner.
template <class T, int LPR>
struct Lane {
  static constexpr int E = kHeld<T>;
  int dim, slot;          // first dim; lane of the wave
  int partner[E];
  int axis[E];
  float sign[E];
  double freq[E];

  __device__ __forceinline__ Lane(const RopeArgs& a, int lane) {
    const int l = lane % LPR;
    dim = l * E;
    slot = lane;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      int i = dim + j, o = 0, f = 0;
      partner[j] = j * 64 + lane;
      axis[j] = 0;
      sign[j] = 0.f;
      freq[j] = 0.0;
      for (int x = 0; x < a.axes; ++x) {
        const int n = a.rot[x] / 2;
        if (i >= o && i < o + 2 * n) {
          const bool second = i >= o + n;
          const int p = second ? i - n : i + n;
          partner[j] = (p % E) * 64 + lane - l + p / E;
          axis[j] = x;
          sign[j] = second ? 1.f : -1.f;
          freq[j] = a.freqs[f + i - o - (second ? n : 0)] * 0.15915494309189533577;   // / (2 pi)
        }
        o += 2 * n;
        f += n;
      }
    }
  }
  // cos and signed sin of the token's angles
  __device__ __forceinline__ void angles(const RopeArgs& a, int64_t b, int64_t n, float (&c)[E],
                                         float (&s)[E]) const {
    double pos[3];
#pragma unroll
    for (int x = 0; x < 3; ++x)
      pos[x] = !a.pos ? (double)(a.pos0 + n)
               : x < a.axes ? (double)a.pos[b * a.pos_bs + n * a.axes + x] : 0.0;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const double t = (axis[j] == 0 ? pos[0] : axis[j] == 1 ? pos[1] : pos[2]) * freq[j];
      const float u = (float)(t - __builtin_rint(t));
      float sn, cs;
      sincospif(2.f * u, &sn, &cs);
      c[j] = cs;
      s[j] = sn * sign[j];
    }
  }
};

// y turned by the angles (s signed for the direction); xch: the wave's E x 64 floats
template <int E>
__device__ __forceinline__ void turn(float (&y)[E], const float (&c)[E], const float (&s)[E],
                                     const int (&partner)[E], int lane, float* xch, float dir) {
#pragma unroll
  for (int j = 0; j < E; ++j) xch[j * 64 + lane] = y[j];
  __builtin_amdgcn_wave_barrier();
  float z[E];
#pragma unroll
  for (int j = 0; j < E; ++j) z[j] = xch[partner[j]];
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < E; ++j) y[j] = __builtin_fmaf(y[j], c[j], dir * z[j] * s[j]);
}

template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// A wave takes 64 / LPR tokens at a time and the heads [h0, h1) of its share (blockIdx.y).
template <class T, int LPR, bool VEC>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeArgs a) {
  constexpr int E = kHeld<T>, kTok = 64 / LPR;
  __shared__ float lds[kWaves][E * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* const xch = lds[wave];
  const Lane<T, LPR> L(a, lane);
  const int total = a.H + 2 * a.Hkv;
  const int h0 = (int)((int64_t)total * blockIdx.y / gridDim.y);
  const int h1 = (int)((int64_t)total * (blockIdx.y + 1) / gridDim.y);
  float w[2][E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const bool in = L.dim + j < a.d;
    w[0][j] = a.qw && in ? a.qw[L.dim + j] : 1.f;
    w[1][j] = a.kw && in ? a.kw[L.dim + j] : 1.f;
  }
  const float inv_d = 1.f / (float)a.d;
  const int64_t rows = a.B * a.N;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * kTok; t0 < rows;
       t0 += (int64_t)gridDim.x * kWaves * kTok) {
    const int64_t row = min(t0 + lane / LPR, rows - 1);   // lanes past the end repeat the last token
    const bool live = t0 + lane / LPR < rows;
    const int64_t b = row / a.N, n = row % a.N;
    const T* src = (const T*)a.x + b * a.bs + n * a.ts;
    float c[E], s[E];
    L.angles(a, b, n, c, s);
    for (int hb = h0; hb < h1; hb += kBatch) {
      float x[kBatch][E];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        load_row<T, VEC>(src + (int64_t)min(hb + u, h1 - 1) * a.d, L.dim, a.d, x[u]);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = hb + u;
        if (h >= h1) break;
        T* dst;
        if (h < a.H + a.Hkv) {
          const bool key = h >= a.H;
          float ss = 0.f;
#pragma unroll
          for (int j = 0; j < E; ++j) ss = __builtin_fmaf(x[u][j], x[u][j], ss);
          const float r = rsqrtf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
#pragma unroll
          for (int j = 0; j < E; ++j) x[u][j] *= r * (key ? w[1][j] : w[0][j]);
          turn(x[u], c, s, L.partner, lane, xch, 1.f);
          dst = key ? (T*)a.k + ((b * a.Hkv + h - a.H) * a.N + n) * a.d
                    : (T*)a.q + ((b * a.H + h) * a.N + n) * a.d;
        } else {
          dst = (T*)a.v + ((b * a.Hkv + h - a.H - a.Hkv) * a.N + n) * a.d;
        }
        if (live) store_row<T, VEC>(dst, L.dim, a.d, x[u]);
      }
    }
  }
}

// kHeld<T> dims of an fp32 gradient row
template <class T, bool VEC>
__device__ __forceinline__ void load_grad(const float* p, int dim, int d, float (&x)[kHeld<T>]) {
#pragma unroll
  for (int j = 0; j < kHeld<T>; j += 4) {
    if constexpr (VEC) {
      f32x4 v = {};
      if (dim + j < d) v = *reinterpret_cast<const f32x4*>(p + dim + j);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j + i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j + i] = dim + j + i < d ? p[dim + j + i] : 0.f;
    }
  }
}

template <class T, int LPR, bool VEC>
__global__ __launch_bounds__(kThreads) void norm_rope_bwd_kernel(RopeArgs a) {
  constexpr int E = kHeld<T>, kTok = 64 / LPR;
  constexpr int kB = kBatch / 2;
  __shared__ float lds[kWaves][E * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* const xch = lds[wave];
  const Lane<T, LPR> L(a, lane);
  const int total = a.H + 2 * a.Hkv;
  const int h0 = (int)((int64_t)total * blockIdx.y / gridDim.y);
  const int h1 = (int)((int64_t)total * (blockIdx.y + 1) / gridDim.y);
  float w[2][E], dw[2][E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const bool in = L.dim + j < a.d;
    w[0][j] = a.qw && in ? a.qw[L.dim + j] : 1.f;
    w[1][j] = a.kw && in ? a.kw[L.dim + j] : 1.f;
    dw[0][j] = dw[1][j] = 0.f;
  }
  const float inv_d = 1.f / (float)a.d;
  const int64_t rows = a.B * a.N;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * kTok; t0 < rows;
       t0 += (int64_t)gridDim.x * kWaves * kTok) {
    const int64_t row = min(t0 + lane / LPR, rows - 1);
    const bool live = t0 + lane / LPR < rows;
    const int64_t b = row / a.N, n = row % a.N;
    const T* src = (const T*)a.x + b * a.bs + n * a.ts;
    T* dst = (T*)a.dx + row * total * a.d;
    float c[E], s[E];
    L.angles(a, b, n, c, s);
    for (int hb = h0; hb < h1; hb += kB) {
      float x[kB][E], g[kB][E];
#pragma unroll
      for (int u = 0; u < kB; ++u) {
        const int h = min(hb + u, h1 - 1);
        const float* gp = h < a.H            ? a.dq + ((b * a.H + h) * a.N + n) * a.d
                          : h < a.H + a.Hkv ? a.dk + ((b * a.Hkv + h - a.H) * a.N + n) * a.d
                                            : a.dv + ((b * a.Hkv + h - a.H - a.Hkv) * a.N + n) * a.d;
        load_grad<T, VEC>(gp, L.dim, a.d, g[u]);
        if (h < a.H + a.Hkv) load_row<T, VEC>(src + (int64_t)h * a.d, L.dim, a.d, x[u]);
      }
#pragma unroll
      for (int u = 0; u < kB; ++u) {
        const int h = hb + u;
        if (h >= h1) break;
        if (h < a.H + a.Hkv) {
          const bool key = h >= a.H;
          turn(g[u], c, s, L.partner, lane, xch, -1.f);
          float ss = 0.f, sg = 0.f;
#pragma unroll
          for (int j = 0; j < E; ++j) {
            ss = __builtin_fmaf(x[u][j], x[u][j], ss);
            sg = __builtin_fmaf(g[u][j] * (key ? w[1][j] : w[0][j]), x[u][j], sg);
          }
          const float r = rsqrtf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
          const float m = row_sum<LPR>(sg) * inv_d * r * r;   // mean(g w x r) r
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float d = g[u][j] * x[u][j] * r;
            if (live) {
              dw[0][j] += key ? 0.f : d;
              dw[1][j] += key ? d : 0.f;
            }
            g[u][j] = r * (g[u][j] * (key ? w[1][j] : w[0][j])) - x[u][j] * r * m;
          }
        }
        if (live) store_row<T, VEC>(dst + (int64_t)h * a.d, L.dim, a.d, g[u]);
      }
    }
  }
  // the workgroup's sums: over the tokens of a wave, then over the waves
  if (!a.part) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int j = 0; j < E; ++j)
#pragma unroll
      for (int off = LPR; off < 64; off <<= 1) dw[which][j] += __shfl_xor(dw[which][j], off, 64);
    __syncthreads();
    if (lane < LPR) {
#pragma unroll
      for (int j = 0; j < E; ++j) xch[lane * E + j] = dw[which][j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.d; i += kThreads) {
      float t = 0.f;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) t += lds[x][i];
      a.part[(((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 + which) * a.d + i] = t;
    }
  }
}

// Sums of the workgroups' parts [parts, 2, d] in their order: 32 columns x 32 groups of parts to a
// workgroup.
__global__ __launch_bounds__(1024) void weight_grad_kernel(const float* __restrict__ part, int parts,
                                                           int d, float* __restrict__ dqw,
                                                           float* __restrict__ dkw) {
  __shared__ float lds[32][33];
  const int cl = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + cl;
  const int per = (parts + 31) / 32;
  float t = 0.f;
  if (col < 2 * d) {
    const int hi = min(parts, (grp + 1) * per);
#pragma unroll 8
    for (int p = grp * per; p < hi; ++p) t += part[(int64_t)p * 2 * d + col];
  }
  lds[grp][cl] = t;
  __syncthreads();
  if (grp == 0 && col < 2 * d) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += lds[i][cl];
    if (col < d && dqw) dqw[col] = s;
    if (col >= d && dkw) dkw[col - d] = s;
  }
}

template <class T, int LPR, bool VEC>
hipError_t launch(const RopeArgs& a, bool bwd) {
  const RopeGrid g = rope_grid(a.B * a.N, a.H + 2 * a.Hkv, 64 / LPR, bwd);
  const dim3 grid((uint32_t)g.x, (uint32_t)g.y);
  if (!bwd) {
    hipLaunchKernelGGL((norm_rope_kernel<T, LPR, VEC>), grid, dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((norm_rope_bwd_kernel<T, LPR, VEC>), grid, dim3(kThreads), 0, a.stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(weight_grad_kernel, dim3((2 * a.d + 31) / 32), dim3(1024), 0, a.stream, a.part,
                     (int)(g.x * g.y), a.d, a.dqw, a.dkw);
  return hipGetLastError();
}

template <int LPR>
hipError_t launch_f32(const RopeArgs& a, bool bwd) {
  return a.vec ? launch<float, LPR, true>(a, bwd) : launch<float, LPR, false>(a, bwd);
}

}  // namespace

hipError_t launch_norm_rope(const RopeArgs& a, bool bwd) {
  if (a.bf16)
    return a.d == 128 ? launch<__bf16, 16, true>(a, bwd) : launch<__bf16, 8, true>(a, bwd);
  switch (rope_lanes(a.d, false)) {
    case 1: return launch_f32<1>(a, bwd);
    case 2: return launch_f32<2>(a, bwd);
    case 4: return launch_f32<4>(a, bwd);
    case 8: return launch_f32<8>(a, bwd);
    case 16: return launch_f32<16>(a, bwd);
    default: return launch_f32<32>(a, bwd);
  }
}

}  // namespace ringx
