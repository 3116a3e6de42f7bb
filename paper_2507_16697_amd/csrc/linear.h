// What the kernels of the linear layer share: the activations with their derivatives, and what becomes of a
// product's values on their way out (bias, activation, residual, the layout).
#pragma once

#include "ringx.h"
#include "ringx_device.h"
#include "ringx_kernels.h"

#include <type_traits>

namespace ringx {

// The standard normal distribution at z and its density's exponential e = exp(-z^2 / 2).  The error
// function by Abramowitz and Stegun 7.1.26 (1.5e-7 off at most), whose exponential is the density's: the
// lower tail comes as a product, without a difference.  So z times it is at most 2.3e-7 off below 0; relative to
// itself 7e-7 down to -1, 4e-6 to -2, 5e-5 to -3, 5e-4 to -4, 4e-3 to -6.  (fp32's z (1 + erf) / 2, whose sum is a
// difference there: 2e-7, 1e-6, 1e-5, 5e-4, and no digit below -5.)  bf16's step is 4e-3.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.f));
  e = fast_exp2(-kLog2e * x * x);
  float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  p = __builtin_fmaf(p, t, 1.421413741f);
  p = __builtin_fmaf(p, t, -0.284496736f);
  p = __builtin_fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * e;
  return z < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * z));
}

constexpr float kTanhA = 1.5957691216057308f;   // 2 sqrt(2 / pi): (1 + tanh u) / 2 = sigmoid(2 u)
constexpr float kTanhB = 0.044715f;

__device__ __forceinline__ float activate(float z, int act) {
  float e;
  switch (act) {
    case RINGX_ACT_GELU: return z * normal_cdf(z, e);
    case RINGX_ACT_GELU_TANH: return z * sigmoid(kTanhA * z * __builtin_fmaf(kTanhB * z, z, 1.f));
    case RINGX_ACT_SILU: return z * sigmoid(z);
  }
  return z;
}

// 16 values of a lane: the choice is made once
__device__ __forceinline__ void activate_all(f32x4 (&x)[4], int act) {
  const auto each = [&](auto f) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[b][e] = f(x[b][e]);
  };
  if (act == RINGX_ACT_GELU) each([](float z) { return activate(z, RINGX_ACT_GELU); });
  else if (act == RINGX_ACT_GELU_TANH) each([](float z) { return activate(z, RINGX_ACT_GELU_TANH); });
  else each([](float z) { return activate(z, RINGX_ACT_SILU); });
}

__device__ __forceinline__ float activate_grad(float z, int act) {
  switch (act) {
    case RINGX_ACT_GELU: {
      float e;
      const float p = normal_cdf(z, e);
      return __builtin_fmaf(z * 0.39894228040143268f, e, p);
    }
    case RINGX_ACT_GELU_TANH: {
      const float g = sigmoid(kTanhA * z * __builtin_fmaf(kTanhB * z, z, 1.f));
      const float y = fminf(fmaxf(z, -32.f), 32.f);   // g (1 - g) is 0 long before: no 0 times infinity
      return __builtin_fmaf(y * g * (1.f - g), kTanhA * __builtin_fmaf(3.f * kTanhB * y, y, 1.f), g);
    }
    case RINGX_ACT_SILU: {
      const float g = sigmoid(z);
      return g * __builtin_fmaf(z, 1.f - g, 1.f);
    }
  }
  return 1.f;
}

// g *= act'(z), the choice made once
template <int U, int N>
__device__ __forceinline__ void grad_all(float (&g)[U][N], const float (&z)[U][N], int act) {
  const auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) g[u][e] *= f(z[u][e]);
  };
  if (act == RINGX_ACT_GELU) each([](float v) { return activate_grad(v, RINGX_ACT_GELU); });
  else if (act == RINGX_ACT_GELU_TANH) each([](float v) { return activate_grad(v, RINGX_ACT_GELU_TANH); });
  else each([](float v) { return activate_grad(v, RINGX_ACT_SILU); });
}

// N neighbouring values from p on, as fp32: N values' 8- or 16-byte pieces (VEC), else the first `n`.
template <int N, bool VEC, class T>
__device__ __forceinline__ void load_values(const T* p, int n, float (&x)[N]) {
  if constexpr (VEC) {
    constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 y = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = y[j];
      }
    } else {
      const u32x2 y = *reinterpret_cast<const u32x2*>(p);
      w[0] = y[0], w[1] = y[1];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (std::is_same_v<T, float>) x[j] = __uint_as_float(w[j]);
      else x[j] = j % 2 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < n ? (float)p[j] : 0.f;
  }
}
template <int N, bool VEC, class T>
__device__ __forceinline__ void store_values(T* p, int n, const float (&x)[N]) {
  if constexpr (VEC) {
    constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      if constexpr (std::is_same_v<T, float>) w[j] = __float_as_uint(x[j]);
      else w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
    }
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i)
        reinterpret_cast<u32x4*>(p)[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    } else {
      *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) p[j] = (T)x[j];
  }
}

// Values (i, j0 .. j0 + N) of a product, n <= N of them inside, to where they go.  b: the bias of these
// columns.  VEC: all N inside and every address a multiple of the piece.
template <int N, bool VEC, class T>
__device__ __forceinline__ void finish(const GemmOut& o, int64_t i, int64_t j0, int n, const float (&b)[N],
                                       float (&x)[N]) {
  const int64_t at = i * o.J + j0;
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] += b[j];
  if (o.pre) store_values<N, VEC>((T*)o.pre + at, n, x);
  if (o.act != RINGX_ACT_NONE) {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = activate(x[j], o.act);
  }
  if (o.residual) {
    float r[N];
    load_values<N, VEC>((const T*)o.residual + at, n, r);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] += r[j];
  }
  if (o.f32) {
    float* const p = (float*)o.out + at;
    if (o.accumulate) {
      float r[N];
      load_values<N, VEC>(p, n, r);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] += r[j];
    }
    store_values<N, VEC>(p, n, x);
  } else if (o.heads) {
    // [.., heads, tokens, d]
    const uint32_t b0 = (uint32_t)i / (uint32_t)o.tokens, t = (uint32_t)i - b0 * (uint32_t)o.tokens;
    if constexpr (VEC) {
      const uint32_t h = (uint32_t)j0 / (uint32_t)o.d, c = (uint32_t)j0 - h * (uint32_t)o.d;
      store_values<N, VEC>((T*)o.out + (((int64_t)b0 * o.heads + h) * o.tokens + t) * o.d + c, n, x);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint32_t h = (uint32_t)(j0 + j) / (uint32_t)o.d, c = (uint32_t)(j0 + j) - h * (uint32_t)o.d;
        if (j < n) ((T*)o.out)[(((int64_t)b0 * o.heads + h) * o.tokens + t) * o.d + c] = (T)x[j];
      }
    }
  } else {
    store_values<N, VEC>((T*)o.out + at, n, x);
  }
}

// Sums of 64 columns of parts, by WAVES waves of a workgroup: a wave every so many parts, then the waves in their
// order.
template <int WAVES>
__device__ __forceinline__ void sum_columns(const ColumnSums& a, uint32_t id, float (*lds)[64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)id * 64 + lane;
  float t = 0.f;
  if (col < a.cols) {
    if (a.rows) {
      // the gradient's own rows
      const auto add = [&](const auto* p) {
#pragma unroll 8
        for (int i = wave; i < a.parts; i += WAVES) t += (float)p[i * a.cols + col];
      };
      if (a.rows_bf16) add((const __bf16*)a.rows);
      else add((const float*)a.rows);
    } else {
#pragma unroll 8
      for (int i = wave; i < a.parts; i += WAVES) t += a.part[i * a.cols + col];
    }
  }
  lds[wave][lane] = t;
  __syncthreads();
  if (wave == 0 && col < a.cols) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += lds[i][lane];
    float* const out = a.out[0] + col;
    *out = a.accumulate ? *out + s : s;
  }
}

}  // namespace ringx
