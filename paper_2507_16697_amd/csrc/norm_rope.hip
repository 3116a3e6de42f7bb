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
// 0.03 of a radian.  The fraction, at most half a turn, is rounded to 32 bits (2^-26 of a turn, 9.4e-8 of a
// radian) and its cosine and sine are the hardware's, two instructions (1.25e-7 off): fp32 rows are off by
// 7.9e-8 rms of their size against 64 bits, by 6.9e-8 with cosines and sines in 64 bits throughout.

#include "ringx_device.h"
#include "ringx_kernels.h"

#include <algorithm>
#include <type_traits>

namespace ringx {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Rows of a lane at work, and in flight behind them, forward: 165 us over 32768 tokens of 48 heads of 128
// (4.9 TB/s; 174 through the caches; without norm and rotation, the copy to the other layout alone took
// 180 in a form without loads ahead).  Without loads ahead, four rows one after the other: 252.
constexpr int kBatch = 2;

// Dims per lane: 16 bytes of the storage type.
template <class T>
constexpr int kHeld = std::is_same_v<T, float> ? 4 : 8;

// kHeld dims of a row as they are stored: 16-byte accesses (VEC), else one by one where dim < d.
// STREAM: past the caches, for tensors that they would not hold anyway.
template <class T, bool VEC, bool STREAM>
__device__ __forceinline__ u32x4 load_raw(const T* p, int dim, int d) {
  u32x4 w = {};
  if constexpr (VEC) {
    const u32x4* const x = reinterpret_cast<const u32x4*>(p + dim);
    if (dim < d) w = STREAM ? __builtin_nontemporal_load(x) : *x;
  } else {
    static_assert(std::is_same_v<T, float>, "bf16 rows come in 16-byte pieces");
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = dim + j < d ? __float_as_uint(p[dim + j]) : 0u;
  }
  return w;
}
template <class T>
__device__ __forceinline__ void unpack(const u32x4& w, float (&x)[kHeld<T>]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (std::is_same_v<T, float>) {
      x[j] = __uint_as_float(w[j]);
    } else {
      x[2 * j] = bf16_lo(w[j]);
      x[2 * j + 1] = bf16_hi(w[j]);
    }
  }
}
template <class T, bool VEC, bool STREAM>
__device__ __forceinline__ void store_raw(T* p, int dim, int d, const u32x4& w) {
  if constexpr (VEC) {
    u32x4* const x = reinterpret_cast<u32x4*>(p + dim);
    if (dim < d) {
      if constexpr (STREAM) __builtin_nontemporal_store(w, x);
      else *x = w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (dim + j < d) p[dim + j] = __uint_as_float(w[j]);
  }
}
template <class T, bool VEC, bool STREAM>
__device__ __forceinline__ void store_row(T* p, int dim, int d, const float (&x)[kHeld<T>]) {
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (std::is_same_v<T, float>) w[j] = __float_as_uint(x[j]);
    else w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
  }
  store_raw<T, VEC, STREAM>(p, dim, d, w);
}

// What rotation needs to know.  Once per workgroup, a word for every dim: the other dim of its pair,
// the pair, whether it is the second of the two, whether it is rotated at all.  Once per token, by the
// wave that holds it, the cosine and sine of every pair.  Lanes then pick those of the dims that they
// hold.  (Formed by every lane for its dims, twice for a pair and with the search for the section
// repeated, they took 25 us of 188 over 32768 tokens of 128-dim heads.)
template <class T, int LPR>
struct Rotation {
  static constexpr int E = kHeld<T>, kTok = 64 / LPR, kDims = E * LPR, kPairs = kDims / 2;
  int dim[kDims];                      // other dim | pair << 8 | second << 16 | rotated << 17
  f32x2 cs[kWaves][kTok][kPairs];

  // before a barrier; all threads
  __device__ __forceinline__ void fill(const RopeArgs& a) {
    for (int i = threadIdx.x; i < kDims; i += kThreads) {
      int x = i, o = 0;
#pragma unroll
      for (int s = 0; s < 3; ++s) {
        const int n = a.rot[s] / 2;
        if (i >= o && i < o + 2 * n) {
          const int second = i >= o + n;
          x = (second ? i - n : i + n) | (o / 2 + (i - o) - second * n) << 8 | second << 16 | 1 << 17;
        }
        o += 2 * n;
      }
      dim[i] = x;
    }
  }
  // the wave's tokens t0 .. (those past the end: the last); the wave reads its own part afterwards
  __device__ __forceinline__ void angles(const RopeArgs& a, int64_t t0, int64_t rows, int wave,
                                         int lane) {
    const int p0 = a.rot[0] / 2, p1 = p0 + a.rot[1] / 2, pairs = p1 + a.rot[2] / 2;
    // a power of two of lanes takes a token's pairs; the others further tokens
    int log2 = 0;
    while ((1 << log2) < pairs && log2 < 6) ++log2;
    for (int p = lane & ((1 << log2) - 1); p < pairs; p += 64) {
      const double f = a.freqs[p] * 0.15915494309189533577;   // turns: / (2 pi)
      const int axis = (p >= p0) + (p >= p1);
      for (int k = lane >> log2; k < kTok; k += 64 >> log2) {
        const int64_t t = min(t0 + k, rows - 1);
        int64_t b = 0, n = t;
        if (a.B > 1) b = t / a.N, n = t - b * a.N;
        const double pos =
            a.pos ? (double)a.pos[b * a.pos_bs + n * a.axes + axis] : (double)(a.pos0 + n);
        const double turns = pos * f;
        const float u = (float)(turns - __builtin_rint(turns));
        // the hardware's cosine and sine, of turns: at most 1.25e-7 off over [-1/2, 1/2]
        cs[wave][k][p] = f32x2{__builtin_amdgcn_cosf(u), __builtin_amdgcn_sinf(u)};
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  // cos and sin, the latter signed for a dim's part in its pair, of the lane's dims
  __device__ __forceinline__ void get(int wave, int lane, float (&c)[E], float (&s)[E]) const {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int x = dim[lane % LPR * E + j];
      const f32x2 y = cs[wave][lane / LPR][x >> 8 & 127];
      const bool on = x >> 17;
      c[j] = on ? y[0] : 1.f;
      s[j] = !on ? 0.f : x >> 16 & 1 ? y[1] : -y[1];
    }
  }
  // where the other members of its pairs lie in a block of E x 64 floats
  __device__ __forceinline__ void partners(int lane, int (&partner)[E]) const {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int p = dim[lane % LPR * E + j] & 255;
      partner[j] = p % E * 64 + lane / LPR * LPR + p / E;
    }
  }
};

// the lane's weights of queries and keys (1 where there are none)
template <class T, bool VEC>
__device__ __forceinline__ void load_weights(const RopeArgs& a, int dim, float (&w)[2][kHeld<T>]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float* p = i == 0 ? a.qw : a.kw;
#pragma unroll
    for (int j = 0; j < kHeld<T>; j += 4) {
      f32x4 x = {1.f, 1.f, 1.f, 1.f};
      if (p) {
        if constexpr (VEC) {
          if (dim + j < a.d) x = *reinterpret_cast<const f32x4*>(p + dim + j);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = dim + j + e < a.d ? p[dim + j + e] : 1.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i][j + e] = x[e];
    }
  }
}

// Rows y[0 .. R) turned by the angles (s signed, dir for the direction); xch: R blocks of E x 64 floats
// of the wave, for the other members of the pairs.
template <int R, int E>
__device__ __forceinline__ void turn(float (&y)[R][E], const float (&c)[E], const float (&s)[E],
                                     const int (&partner)[E], int lane, float* xch, float dir) {
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int j = 0; j < E; ++j) xch[(u * E + j) * 64 + lane] = y[u][j];
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int u = 0; u < R; ++u) {
    float z[E];
#pragma unroll
    for (int j = 0; j < E; ++j) z[j] = xch[u * E * 64 + partner[j]];
#pragma unroll
    for (int j = 0; j < E; ++j) y[u][j] = __builtin_fmaf(y[u][j], c[j], dir * z[j] * s[j]);
  }
  __builtin_amdgcn_wave_barrier();
}

// Sum over the LPR lanes of a row, in every one of them: lane exchanges within 16 lanes are part of the
// add itself.
template <int CTRL>
__device__ __forceinline__ float add_lane(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  if constexpr (LPR >= 2) x = add_lane<0xB1>(x);     // lanes 1 0 3 2 of every four
  if constexpr (LPR >= 4) x = add_lane<0x4E>(x);     // lanes 2 3 0 1
  if constexpr (LPR >= 8) x = add_lane<0x141>(x);    // mirrored in eight: the other four
  if constexpr (LPR >= 16) x = add_lane<0x140>(x);   // mirrored in sixteen: the other eight
  if constexpr (LPR >= 32) x += __shfl_xor(x, 16, 64);
  return x;
}

// A wave takes 64 / LPR tokens and the heads [h0, h1) of its share (blockIdx.y), kBatch rows of a lane
// at a time while the next ones arrive.
template <class T, int LPR, bool VEC, bool STREAM>
__global__ __launch_bounds__(kThreads, 4) void norm_rope_kernel(RopeArgs a) {
  constexpr int E = kHeld<T>, kTok = 64 / LPR;
  __shared__ float lds[kWaves][kBatch * E * 64];
  __shared__ Rotation<T, LPR> rotation;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const xch = lds[wave];
  const int total = a.H + 2 * a.Hkv, turned = a.H + a.Hkv;
  const int h0 = (int)((int64_t)total * blockIdx.y / gridDim.y);
  const int h1 = (int)((int64_t)total * (blockIdx.y + 1) / gridDim.y);
  const int64_t rows = a.B * a.N;
  const int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * kTok + lane / LPR;
  const bool live = t < rows;
  const int64_t row = live ? t : rows - 1;   // lanes past the end repeat the last token
  const int64_t b = row / a.N, n = row % a.N;
  const T* src = (const T*)a.x + b * a.bs + n * a.ts;
  const int dim = lane % LPR * E;
  u32x4 raw[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u)
    raw[u] = load_raw<T, VEC, STREAM>(src + (int64_t)min(h0 + u, h1 - 1) * a.d, dim, a.d);

  rotation.fill(a);
  __syncthreads();
  int partner[E];
  float c[E], s[E], w[2][E];
  load_weights<T, VEC>(a, dim, w);
  rotation.angles(a, t - lane / LPR, rows, wave, lane);
  rotation.get(wave, lane, c, s);
  rotation.partners(lane, partner);
  const float inv_d = 1.f / (float)a.d;
  T* const q = (T*)a.q + (b * a.H * a.N + n) * a.d;
  T* const k = (T*)a.k + (b * a.Hkv * a.N + n) * a.d;
  T* const v = (T*)a.v + (b * a.Hkv * a.N + n) * a.d;
  const int64_t head = a.N * a.d;   // elements of an output head
  for (int hb = h0; hb < h1; hb += kBatch) {
    u32x4 next[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      next[u] = load_raw<T, VEC, STREAM>(src + (int64_t)min(hb + kBatch + u, h1 - 1) * a.d, dim, a.d);
    if (hb < turned) {
      float x[kBatch][E];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        unpack<T>(raw[u], x[u]);
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) ss = __builtin_fmaf(x[u][j], x[u][j], ss);
        const float r = rsqrtf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
        const bool key = hb + u >= a.H;
#pragma unroll
        for (int j = 0; j < E; ++j) x[u][j] *= r * (key ? w[1][j] : w[0][j]);
      }
      turn(x, c, s, partner, lane, xch, 1.f);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = hb + u;
        if (live && h < h1 && h < turned)
          store_row<T, VEC, STREAM>(h < a.H ? q + h * head : k + (h - a.H) * head, dim, a.d, x[u]);
      }
    }
    if (hb + kBatch > turned) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = hb + u;
        if (live && h < h1 && h >= turned) store_raw<T, VEC, STREAM>(v + (h - turned) * head, dim, a.d, raw[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) raw[u] = next[u];
  }
}

// kHeld<T> dims of an fp32 gradient row
template <class T, bool VEC, bool STREAM>
__device__ __forceinline__ void load_grad(const float* p, int dim, int d, float (&x)[kHeld<T>]) {
#pragma unroll
  for (int j = 0; j < kHeld<T>; j += 4) {
    if constexpr (VEC) {
      f32x4 v = {};
      const f32x4* const y = reinterpret_cast<const f32x4*>(p + dim + j);
      if (dim + j < d) v = STREAM ? __builtin_nontemporal_load(y) : *y;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j + i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j + i] = dim + j + i < d ? p[dim + j + i] : 0.f;
    }
  }
}

// One row at a time and four waves on a SIMD, whose loads cover each other: 320 us over 32768 tokens of 48
// heads of 128 (5.0 TB/s; a copy of that size reaches 5.4).  Loading the next row ahead takes the
// registers of a wave (326 us, and 87 against 79 over 8192 tokens, whose loads hit the caches), two rows at
// a time too (340).
template <class T, int LPR, bool VEC, bool STREAM>
__global__ __launch_bounds__(kThreads, 4) void norm_rope_bwd_kernel(RopeArgs a) {
  constexpr int E = kHeld<T>, kTok = 64 / LPR;
  __shared__ float lds[kWaves][E * 64];
  __shared__ Rotation<T, LPR> rotation;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const xch = lds[wave];
  const int dim = lane % LPR * E;
  rotation.fill(a);
  __syncthreads();
  int partner[E];
  rotation.partners(lane, partner);
  const int total = a.H + 2 * a.Hkv;
  const int h0 = (int)((int64_t)total * blockIdx.y / gridDim.y);
  const int h1 = (int)((int64_t)total * (blockIdx.y + 1) / gridDim.y);
  float w[2][E], dw[2][E];
  load_weights<T, VEC>(a, dim, w);
#pragma unroll
  for (int j = 0; j < E; ++j) dw[0][j] = dw[1][j] = 0.f;
  const float inv_d = 1.f / (float)a.d;
  const int64_t rows = a.B * a.N, head = a.N * a.d;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * kTok; t0 < rows;
       t0 += (int64_t)gridDim.x * kWaves * kTok) {
    const bool live = t0 + lane / LPR < rows;
    const int64_t row = live ? t0 + lane / LPR : rows - 1;
    const int64_t b = row / a.N, n = row % a.N;
    const T* src = (const T*)a.x + b * a.bs + n * a.ts;
    T* dst = (T*)a.dx + row * total * a.d;
    float c[E], s[E];
    rotation.angles(a, t0, rows, wave, lane);
    rotation.get(wave, lane, c, s);
    // heads [lo, hi) of the queries or keys, whose gradients start at gp and which are columns
    // `first` .. of a token's heads
    auto normed = [&](int lo, int hi, int first, const float* gp, const float (&w)[E],
                      float (&dw)[E]) {
      for (int h = lo; h < hi; ++h) {
        float x[E], g[1][E];
        load_grad<T, VEC, STREAM>(gp + h * head, dim, a.d, g[0]);
        unpack<T>(load_raw<T, VEC, STREAM>(src + (int64_t)(first + h) * a.d, dim, a.d), x);
        turn(g, c, s, partner, lane, xch, -1.f);
        float ss = 0.f, sg = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
          ss = __builtin_fmaf(x[j], x[j], ss);
          sg = __builtin_fmaf(g[0][j] * w[j], x[j], sg);
        }
        const float r = rsqrtf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
        const float m = row_sum<LPR>(sg) * inv_d * r * r;   // mean(g w x r) r
        const float count = live ? r : 0.f;                  // a repeated token adds nothing
        float dx[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
          dw[j] = __builtin_fmaf(g[0][j] * x[j], count, dw[j]);
          dx[j] = r * (g[0][j] * w[j]) - x[j] * r * m;
        }
        if (live) store_row<T, VEC, STREAM>(dst + (int64_t)(first + h) * a.d, dim, a.d, dx);
      }
    };
    normed(h0, min(h1, a.H), 0, a.dq + (b * a.H * a.N + n) * a.d, w[0], dw[0]);
    normed(max(h0 - a.H, 0), min(h1 - a.H, a.Hkv), a.H, a.dk + (b * a.Hkv * a.N + n) * a.d, w[1],
           dw[1]);
    const float* gv = a.dv + (b * a.Hkv * a.N + n) * a.d;
#pragma unroll 2
    for (int h = max(h0 - a.H - a.Hkv, 0); h < h1 - a.H - a.Hkv; ++h) {
      float g[E];
      load_grad<T, VEC, STREAM>(gv + h * head, dim, a.d, g);
      if (live) store_row<T, VEC, STREAM>(dst + (int64_t)(a.H + a.Hkv + h) * a.d, dim, a.d, g);
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

// Sums of the workgroups' parts [parts, 2, d] in their order: 16 columns x 64 groups of parts to a
// workgroup, 16 loads of a thread in flight, since the loads' latency is all that it waits for.
constexpr int kSumCols = 16, kSumGroups = 64;
__global__ __launch_bounds__(1024) void weight_grad_kernel(const float* __restrict__ part, int parts,
                                                           int d, float* __restrict__ dqw,
                                                           float* __restrict__ dkw) {
  __shared__ float lds[kSumGroups][kSumCols + 1];
  const int cl = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols;
  const int col = blockIdx.x * kSumCols + cl;
  const int per = (parts + kSumGroups - 1) / kSumGroups;
  float t = 0.f;
  if (col < 2 * d) {
    const int hi = min(parts, (grp + 1) * per);
    for (int p = grp * per; p < hi; p += 16) {
      float x[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = part[(int64_t)min(p + u, hi - 1) * 2 * d + col];
#pragma unroll
      for (int u = 0; u < 16; ++u) t += p + u < hi ? x[u] : 0.f;
    }
  }
  lds[grp][cl] = t;
  __syncthreads();
  if (grp == 0 && col < 2 * d) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kSumGroups; ++i) s += lds[i][cl];
    if (col < d && dqw) dqw[col] = s;
    if (col >= d && dkw) dkw[col - d] = s;
  }
}

template <class T, int LPR, bool VEC, bool STREAM>
hipError_t launch(const RopeArgs& a, bool bwd) {
  const RopeGrid g = rope_grid(a.B * a.N, a.H + 2 * a.Hkv, 64 / LPR, bwd);
  const dim3 grid((uint32_t)g.x, (uint32_t)g.y);
  if (!bwd) {
    hipLaunchKernelGGL((norm_rope_kernel<T, LPR, VEC, STREAM>), grid, dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((norm_rope_bwd_kernel<T, LPR, VEC, STREAM>), grid, dim3(kThreads), 0, a.stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(weight_grad_kernel, dim3((2 * a.d + kSumCols - 1) / kSumCols), dim3(kSumCols * kSumGroups), 0, a.stream, a.part,
                     (int)(g.x * g.y), a.d, a.dqw, a.dkw);
  return hipGetLastError();
}

// From 384 MB on, half as much again as the memory-side cache holds, past the caches.  us, as is -> past
// them: forward, 16 heads of 128, 8192 tokens (201 MB) 37 -> 41, 12288 (302) 66 -> 67, 16384 (403) 88 -> 82,
// 32768 (805) 174 -> 165; backward, 16/4 heads of 64, 16384 tokens (201) 43 -> 45, 32768 (403) 85 -> 84, 65536
// (805) 164 -> 157; 16 of 128, 32768 (1611) 324 -> 322.
template <class T, int LPR>
hipError_t launch_vec(const RopeArgs& a, bool bwd) {
  const int64_t values = a.B * a.N * (a.H + 2 * a.Hkv) * a.d;
  const int64_t bytes = values * (2 * (int64_t)sizeof(T) + (bwd ? 4 : 0));
  return bytes >= 384000000 ? launch<T, LPR, true, true>(a, bwd) : launch<T, LPR, true, false>(a, bwd);
}

template <int LPR>
hipError_t launch_f32(const RopeArgs& a, bool bwd) {
  return a.vec ? launch_vec<float, LPR>(a, bwd) : launch<float, LPR, false, false>(a, bwd);
}

}  // namespace

hipError_t launch_norm_rope(const RopeArgs& a, bool bwd) {
  if (a.bf16) return a.d == 128 ? launch_vec<__bf16, 16>(a, bwd) : launch_vec<__bf16, 8>(a, bwd);
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
