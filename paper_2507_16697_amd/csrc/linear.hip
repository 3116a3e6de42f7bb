// The linear layer y = act(x w^T + b) + residual and its backward, around the matrix products of
// gemm_bf16.hip and gemm_f32.hip: the product for a few rows, what joins a split product, the pass over dy
// that gives dz = dy act'(pre) and the bias's gradient, and operands copied to rows that the products take.

#include "linear.h"

#include <algorithm>

namespace ringx {
namespace {

// -------------------------------------------------------------------------------------------------
// A few rows (a token at a time, or some of them), bf16.  Bound by the weights' bytes: every weight is
// loaded once, for v_mfma_f32_16x16x32_bf16 (lane l: row l % 16, r = 8 (l / 16) .. + 7), NB blocks of 16 features
// to a workgroup whose waves take turns along K.  The rows of x, MB blocks of 16 of them (those past M repeat
// the last), come from the caches, once for each workgroup.
//
// VEC: both go through the wave's own LDS, since a fragment's load touches 16 lines at a time and takes four times
// as long as one of whole 64-byte pieces: lane l loads row l / 4 of a block, piece l % 4, XORed with (row / 4) so
// that 16 rows' same piece lies in 16 places.  (Bank conflicts are 3.8 cycles to an LDS instruction all the same; with
// the row's two bits the other way round the times were equal.  LDS is not what it waits for.)  Two buffers: the next
// turn's loads are in flight while a turn is multiplied.  One row of 2048 to 8192: 5.8 us where the memory-side cache
// holds the weights, 9.9 where they come from HBM.

template <int MB, int NB, int WAVES, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(GemmArgs a) {
  constexpr int kBlocks = MB + NB;
  // steps of 32 of K in a turn: what LDS (VEC) or the registers hold
  constexpr int kSteps = VEC ? (kBlocks == 2 ? 4 : kBlocks <= 4 ? 2 : 1) : (MB >= 3 ? 2 : 4);
  constexpr int kTurn = kSteps * kBlocks * 1024, kStage = VEC ? 2 * kTurn : 0, kSums = MB * NB * 1024;   // of a wave
  __shared__ __attribute__((aligned(1024))) char lds[WAVES * (kStage > kSums ? kStage : kSums)];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t j0 = (int64_t)blockIdx.x * (16 * NB);
  const int K = (int)a.R;
  const bool heads = a.P.heads != 0;
  const int row = VEC ? lane >> 2 : n;
  const __bf16 *w[NB], *x[MB];
#pragma unroll
  for (int f = 0; f < NB; ++f) w[f] = (const __bf16*)a.Q.p + min(j0 + 16 * f + row, a.J - 1) * a.Q.ld;
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int64_t i = min((int64_t)(16 * m + row), a.I - 1);
    int64_t at = i * a.P.ld;
    if (heads) {
      const uint32_t b = (uint32_t)i / (uint32_t)a.P.tokens;
      at = (int64_t)b * a.P.tokens * a.P.cols + (i - (int64_t)b * a.P.tokens) * a.P.d;
    }
    x[m] = (const __bf16*)a.P.p + at;
  }
  const auto place = [&](int k) {   // column k of a row of x
    if (!heads) return (int64_t)k;
    const uint32_t h = (uint32_t)k / (uint32_t)a.P.d;
    return (int64_t)h * a.P.tokens * a.P.d + (k - (int)h * (int)a.P.d);
  };
  const auto straight = [](int k) { return (int64_t)k; };
  const auto values = [&](const __bf16* p, int k, auto at) {   // one by one, zeros past K
    bf16x8 v = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const __bf16 y = p[at(min(k + e, K - 1))];
      v[e] = k + e < K ? y : (__bf16)0.f;
    }
    return v;
  };
  f32x4 acc[MB * NB];
#pragma unroll
  for (int m = 0; m < MB * NB; ++m) acc[m] = f32x4{};
  const uint32_t base = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * kStage);
  const int piece = (lane & 3) ^ (lane >> 4), read = wave * kStage + n * 64 + ((g ^ (n >> 2)) << 4);
  const auto load = [&](int k0, uint32_t to) {   // what lies past K repeats what does not
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int k = min(k0 + 32 * u + 8 * piece, K - 8);
#pragma unroll
      for (int f = 0; f < NB; ++f) load_lds16(w[f] + k, to + (u * kBlocks + f) * 1024);
#pragma unroll
      for (int m = 0; m < MB; ++m) load_lds16(x[m] + place(k), to + (u * kBlocks + NB + m) * 1024);
    }
  };
  constexpr int kTurns = WAVES * 32 * kSteps;   // of K, from a wave's turn to its next
  int at = 0;                                   // the turn's buffer
  const int first = wave * 32 * kSteps;
  if constexpr (VEC) {
    if (first < K) load(first, base);           // a short K leaves waves without a turn
  }
  for (int k0 = first; k0 < K; k0 += kTurns) {
    if constexpr (VEC) {
      if (k0 + kTurns < K) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what lies there has been read
        load(k0 + kTurns, base + kTurn - at);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kSteps * kBlocks) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int k = k0 + 32 * u + 8 * g;
      bf16x8 wv[NB], xv[MB];
      if constexpr (VEC) {
        const auto get = [&](int i) {
          const bf16x8 v = *reinterpret_cast<const bf16x8*>(lds + at + read + (u * kBlocks + i) * 1024);
          return k < K ? v : bf16x8{};
        };
#pragma unroll
        for (int f = 0; f < NB; ++f) wv[f] = get(f);
#pragma unroll
        for (int m = 0; m < MB; ++m) xv[m] = get(NB + m);
      } else {
#pragma unroll
        for (int f = 0; f < NB; ++f) wv[f] = values(w[f], k, straight);
#pragma unroll
        for (int m = 0; m < MB; ++m) xv[m] = values(x[m], k, place);
      }
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int f = 0; f < NB; ++f)
          acc[NB * m + f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[f], xv[m], acc[NB * m + f], 0, 0, 0);
    }
    at = kTurn - at;
  }
  f32x4* const sums = reinterpret_cast<f32x4*>(lds) + lane;   // [wave][block][lane]
  // The sums lie where every wave's loads go: none may be in flight, whichever way the wave came here.  The compiler
  // does not wait for loads that are inline assembly.
  if constexpr (VEC) wait_vmem_all();
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MB * NB; ++m) sums[(wave * MB * NB + m) * 64] = acc[m];
  __syncthreads();
  // a wave ends a block at a time: the waves' sums in their order
  for (int m = wave; m < MB * NB; m += WAVES) {
    f32x4 s = sums[m * 64];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s += sums[(i * MB * NB + m) * 64];
    const int64_t i = 16 * (m / NB) + n, j = j0 + 16 * (m % NB) + 4 * g;
    const int inside = (int)max((int64_t)0, min((int64_t)4, a.J - j));
    if (i >= a.I || inside == 0) continue;
    float b[4], y[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = a.o.bias && e < inside ? a.o.bias[j + e] : 0.f;
    if (a.J % 4 == 0) finish<4, true, __bf16>(a.o, i, j, 4, b, y);
    else finish<4, false, __bf16>(a.o, i, j, inside, b, y);
  }
}

template <int MB, int NB, bool VEC>
hipError_t launch_few_rows_as(const GemmArgs& a) {
  const dim3 grid((uint32_t)((a.J + 16 * NB - 1) / (16 * NB)));
  // 4 waves; 8 where there are few workgroups and much of K (us of 8 / 4: one row of 8192 to 2048 8.7 / 10.6, of 2048
  // to 8192 7.8 / 6.5; 64 rows of 2048 to 2048 6.8 / 9.2)
  if constexpr (VEC || MB == 1) {   // others have less of K (linear_few)
    if (grid.x <= 256 && a.R >= 1024) {
      hipLaunchKernelGGL((few_rows_kernel<MB, NB, 8, VEC>), grid, dim3(512), 0, a.stream, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((few_rows_kernel<MB, NB, 4, VEC>), grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

template <bool VEC>
hipError_t launch_few_rows(const GemmArgs& a) {
  if (a.I <= 16) return launch_few_rows_as<1, 1, VEC>(a);
  if constexpr (VEC) {
    // two blocks of features where one to each compute unit does not do (64 rows, us of two / one: 2048 to 6144
    // 9.4 / 11.5, to 8192 10.2 / 12.8, to 4096 9.2 / 8.2)
    if (a.J > 4096) {
      if (a.I <= 32) return launch_few_rows_as<2, 2, VEC>(a);
      if (a.I <= 48) return launch_few_rows_as<3, 2, VEC>(a);
      return launch_few_rows_as<4, 2, VEC>(a);
    }
  }
  if (a.I <= 32) return launch_few_rows_as<2, 1, VEC>(a);
  if (a.I <= 48) return launch_few_rows_as<3, 1, VEC>(a);
  return launch_few_rows_as<4, 1, VEC>(a);
}

// -------------------------------------------------------------------------------------------------
// The parts of a split fp32 product, in their order, then its epilogue.

template <class T, bool VEC>
__global__ __launch_bounds__(256) void join_kernel(GemmArgs a) {
  const int64_t per = (a.J + 3) / 4, total = a.I * per;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
    const int64_t i = t / per, j = (t - i * per) * 4;
    const int inside = (int)min((int64_t)4, a.J - j);
    float x[4] = {}, b[4];
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      float y[4];
      load_values<4, VEC>(a.part + s * a.I * a.J + i * a.J + j, inside, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = a.o.bias && e < inside ? a.o.bias[j + e] : 0.f;
    finish<4, VEC, T>(a.o, i, j, inside, b, x);
  }
}

template <class T>
hipError_t launch_product(const GemmArgs& a) {
  if constexpr (std::is_same_v<T, __bf16>) {
    return launch_gemm_bf16(a);
  } else {
    const hipError_t e = launch_gemm_f32(a);
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t wgs = std::min<int64_t>((a.I * ((a.J + 3) / 4) + 255) / 256, 4096);
    if (a.J % 4 == 0 && a.o.d % 4 == 0)
      hipLaunchKernelGGL((join_kernel<T, true>), dim3((uint32_t)wgs), dim3(256), 0, a.stream, a);
    else
      hipLaunchKernelGGL((join_kernel<T, false>), dim3((uint32_t)wgs), dim3(256), 0, a.stream, a);
    return hipGetLastError();
  }
}

// -------------------------------------------------------------------------------------------------
// An operand copied to rows of `ld` values, zeros behind its columns: bf16 whose rows do not come in 16-byte
// pieces, and heads where a product does not walk them itself.

template <class T>
struct Pack {
  GemmIn x[2];
  T* out[2];
  int64_t ld[2];
  uint32_t wgs[2];   // workgroups; 0: nothing to copy
  bool vec[2];       // in 16-byte pieces
};

template <class T>
__global__ __launch_bounds__(256) void pack_kernel(Pack<T> a) {
  constexpr int N = 16 / (int)sizeof(T);
  const int k = blockIdx.x >= a.wgs[0];
  const GemmIn& x = a.x[k];
  const uint32_t per = (uint32_t)((a.ld[k] + N - 1) / N), wg = k ? blockIdx.x - a.wgs[0] : blockIdx.x;
  const int64_t total = x.rows * per;
  for (int64_t t = (int64_t)wg * 256 + threadIdx.x; t < total; t += (int64_t)a.wgs[k] * 256) {
    // rows of a tensor fit 32 bits, its pieces need not
    const uint32_t i = total >> 32 ? (uint32_t)(t / per) : (uint32_t)t / per;
    const uint32_t c = (uint32_t)(t - (int64_t)i * per) * N;
    int64_t row = (int64_t)i * x.ld;
    if (x.heads) {
      const uint32_t b = i / (uint32_t)x.tokens;
      row = (int64_t)b * x.tokens * x.cols + (int64_t)(i - b * (uint32_t)x.tokens) * x.d;
    }
    const T* const p = (const T*)x.p + row;
    T* const q = a.out[k] + (int64_t)i * a.ld[k] + c;
    auto column = [&](uint32_t j) {
      if (!x.heads) return (int64_t)j;
      const uint32_t h = j / (uint32_t)x.d;
      return (int64_t)h * x.tokens * x.d + (j - h * (uint32_t)x.d);
    };
    if (a.vec[k]) {
      *reinterpret_cast<u32x4*>(q) = *reinterpret_cast<const u32x4*>(p + column(c));
    } else {
      T v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const T y = p[column(min(c + e, (uint32_t)x.cols - 1))];
        v[e] = c + e < x.cols ? y : (T)0.f;
      }
      if (a.ld[k] % N == 0) {
        *reinterpret_cast<u32x4*>(q) = __builtin_bit_cast(u32x4, v);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < a.ld[k]) q[e] = v[e];
      }
    }
  }
}

// Operands x and y as the products take them, copied to the workspace where the plan says so (offset >= 0).
template <class T>
hipError_t pack(GemmIn* x, int64_t at_x, int64_t ld_x, GemmIn* y, int64_t at_y, int64_t ld_y, void* workspace,
                hipStream_t stream) {
  constexpr int N = 16 / (int)sizeof(T);
  Pack<T> a{};
  const int64_t at[2] = {x ? at_x : -1, y ? at_y : -1}, ld[2] = {ld_x, ld_y};
  GemmIn* const in[2] = {x, y};
  for (int k = 0; k < 2; ++k) {
    if (at[k] < 0) continue;
    GemmIn& s = *in[k];
    a.x[k] = s, a.ld[k] = ld[k], a.out[k] = (T*)(static_cast<char*>(workspace) + at[k]);
    a.wgs[k] = (uint32_t)std::min<int64_t>((s.rows * ((ld[k] + N - 1) / N) + 255) / 256, 8192);
    a.vec[k] = ld[k] == s.cols && s.cols % N == 0 && (s.heads ? s.d % N == 0 : s.ld % N == 0);
    s.p = a.out[k], s.heads = 0, s.ld = s.cols = ld[k];
  }
  if (a.wgs[0] + a.wgs[1] == 0) return hipSuccess;
  hipLaunchKernelGGL((pack_kernel<T>), dim3(a.wgs[0] + a.wgs[1]), dim3(256), 0, stream, a);
  return hipGetLastError();
}

// -------------------------------------------------------------------------------------------------
// dz = dy act'(pre), with zeros up to `ld` columns, and parts [gridDim.y, O] of its column sums.  Bound by
// HBM: dy and pre are read and dz written once; the sums are of dz before its rounding.

struct GradPass {
  const void *dy, *pre;   // [M, O]; pre null without an activation
  void* dz;               // [M, ld] or null
  float* part;            // or null
  int64_t M, O, ld, rows; // rows of a workgroup
  int act, across;        // threads across the columns, 8 of them each
};

// A thread's 8 columns lie side by side (VEC), or `across` apart, neighbours in neighbouring lanes.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void grad_pass_kernel(GradPass a) {
  constexpr int U = 2;   // 8194 x 3840 bf16: 38 us, with 4 45 (registers leave fewer waves)
  __shared__ float lds[256 * 9];
  const int c = threadIdx.x % a.across, down = 256 / a.across;
  const int64_t first = (int64_t)blockIdx.x * a.across * 8;
  const int64_t end = min(a.M, (blockIdx.y + 1) * a.rows);
  const auto column = [&](int e) { return VEC ? first + c * 8 + e : first + e * a.across + c; };
  float sum[8] = {};
  if (column(0) < a.ld) {
    for (int64_t r = blockIdx.y * a.rows + threadIdx.x / a.across; r < end; r += U * down) {
      float g[U][8], z[U][8];
      uint32_t gw[U][8], zw[U][8];   // not VEC: as they are stored
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = min(r + u * down, end - 1) * a.O;
        if constexpr (VEC) {
          load_values<8, true>((const T*)a.dy + at + column(0), 8, g[u]);
          if (a.pre) load_values<8, true>((const T*)a.pre + at + column(0), 8, z[u]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint32_t y = 0u, w = 0u;
            if (column(e) < a.O) {
              y = raw_bits((const T*)a.dy + at + column(e));
              if (a.pre) w = raw_bits((const T*)a.pre + at + column(e));
            }
            gw[u][e] = y, zw[u][e] = w;
          }
        }
      }
      if constexpr (!VEC) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) g[u][e] = from_raw<T>(gw[u][e]), z[u][e] = from_raw<T>(zw[u][e]);
      }
      if (a.pre) grad_all(g, z, a.act);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r + u * down >= end) continue;
        if (a.dz) {
          T* const p = (T*)a.dz + (r + u * down) * a.ld;
          if constexpr (VEC) {
            store_values<8, true>(p + column(0), 8, g[u]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (column(e) < a.ld) p[column(e)] = (T)g[u][e];
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += g[u][e];
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) lds[threadIdx.x * 9 + e] = sum[e];
  __syncthreads();
  for (int j = threadIdx.x; j < a.across * 8 && first + j < a.O; j += 256) {
    float s = 0.f;
    const int of = VEC ? j / 8 : j % a.across, e = VEC ? j % 8 : j / a.across;
    for (int d = 0; d < down; ++d) s += lds[(d * a.across + of) * 9 + e];
    a.part[blockIdx.y * a.O + first + j] = s;
  }
}

template <class T>
hipError_t launch_grad_pass(GradPass a, bool few, hipStream_t stream) {
  const GradGrid g = grad_grid(a.M, a.O, few);
  a.across = g.across, a.rows = g.rows;
  const dim3 grid((uint32_t)g.x, (uint32_t)g.y);
  if (a.O % 8 == 0) hipLaunchKernelGGL((grad_pass_kernel<T, true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((grad_pass_kernel<T, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

// -------------------------------------------------------------------------------------------------
// Column sums of parts: 16 columns x 64 groups of parts to a workgroup, 16 loads of a thread in flight,
// since the loads' latency is all that it waits for.

constexpr int kSumCols = 16, kSumGroups = 64;
__global__ __launch_bounds__(1024) void column_sums_kernel(ColumnSums a) {
  __shared__ float lds[kSumGroups][kSumCols + 1];
  const int cl = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols;
  const int64_t col = (int64_t)blockIdx.x * kSumCols + cl;
  const int per = (a.parts + kSumGroups - 1) / kSumGroups;
  float t = 0.f;
  if (col < a.cols) {
    const int hi = min(a.parts, (grp + 1) * per);
    for (int p = grp * per; p < hi; p += 16) {
      float x[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = a.part[(int64_t)min(p + u, hi - 1) * a.cols + col];
#pragma unroll
      for (int u = 0; u < 16; ++u) t += p + u < hi ? x[u] : 0.f;
    }
  }
  lds[grp][cl] = t;
  __syncthreads();
  if (grp == 0 && col < a.cols) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kSumGroups; ++i) s += lds[i][cl];
    float* const p = col < a.split ? a.out[0] : a.out[1];
    if (p) {
      const int64_t j = col < a.split ? col : col - a.split;
      p[j] = a.accumulate ? p[j] + s : s;
    }
  }
}

char* at(void* workspace, int64_t offset) { return static_cast<char*>(workspace) + offset; }

template <class T>
hipError_t forward(const LinearArgs& a) {
  const LinearPlan p = linear_plan(a.s);
  GemmArgs g;
  g.P = a.x(), g.Q = a.weights();
  g.I = a.s.M, g.J = a.s.O, g.R = a.s.K, g.stream = a.stream;
  g.o.out = a.y, g.o.pre = a.pre, g.o.residual = a.residual, g.o.bias = a.bias, g.o.J = a.s.O;
  g.o.act = a.act;
  if constexpr (std::is_same_v<T, __bf16>) {
    if (p.few) return linear_few_pieces(a.s) ? launch_few_rows<true>(g) : launch_few_rows<false>(g);
  }
  const hipError_t e = pack<T>(&g.P, p.x, p.ldx, &g.Q, p.w, p.ldw, a.workspace, a.stream);
  if (e != hipSuccess) return e;
  g.R = p.R;
  g.splits = p.splits, g.side = p.side, g.cut = p.cut, g.part = (float*)at(a.workspace, p.part);
  return launch_product<T>(g);
}

template <class T>
hipError_t backward(const LinearArgs& a) {
  const LinearPlan p = linear_bwd_plan(a.s, a.act);
  hipError_t e = hipSuccess;
  // dz, and the bias's gradient
  GemmIn dz;
  dz.p = a.dy, dz.rows = a.s.M, dz.cols = dz.ld = a.s.O;
  const bool own = p.dz >= 0 && (a.dx || a.dw);
  const bool both = p.pair && a.dx && a.dw;
  const bool rows = a.dbias && both && !own && !a.act && a.s.M <= kRowsSummed;   // summed beside the products
  if (own || (a.dbias && !rows)) {
    GradPass g{};
    g.dy = a.dy, g.pre = a.act ? a.pre : nullptr, g.M = a.s.M, g.O = a.s.O, g.act = a.act;
    g.dz = own ? at(a.workspace, p.dz) : nullptr, g.ld = p.ldz;
    g.part = a.dbias ? (float*)at(a.workspace, p.sums) : nullptr;
    e = launch_grad_pass<T>(g, p.pair, a.stream);
    if (e != hipSuccess) return e;
    if (own) dz.p = g.dz, dz.cols = dz.ld = p.ldz;
  }
  ColumnSums c;
  if (a.dbias) {
    c.part = (float*)at(a.workspace, p.sums), c.parts = (int)grad_grid(a.s.M, a.s.O, p.pair).y;
    if (rows) c.rows = a.dy, c.rows_bf16 = a.s.bf16, c.parts = (int)a.s.M;
    c.cols = c.split = a.s.O, c.out[0] = a.dbias, c.accumulate = a.accumulate, c.stream = a.stream;
    if (!both) e = launch_column_sums(c);
    if (e != hipSuccess) return e;
  }
  GemmArgs x, w;
  x.stream = w.stream = a.stream, x.P = w.P = dz;
  x.Q = a.weights(), w.Q = a.x();
  e = pack<T>(a.dx ? &x.Q : nullptr, p.w, p.ldw, a.dw ? &w.Q : nullptr, p.x, p.ldx, a.workspace, a.stream);
  if (e != hipSuccess) return e;
  if (a.dx) {
    x.q_slow = true;
    x.I = a.s.M, x.J = a.s.K, x.R = dz.cols, x.splits = p.splits_dx, x.side = p.side_dx, x.cut = p.cut_dx;
    x.part = (float*)at(a.workspace, p.part);
    x.o.out = a.dx, x.o.J = a.s.K, x.o.f32 = a.dx_f32 && !a.s.heads;
    if (a.s.heads) x.o.heads = a.s.heads, x.o.tokens = a.s.tokens, x.o.d = a.s.K / a.s.heads;
  }
  if (a.dw) {
    w.p_slow = w.q_slow = true;
    w.I = a.s.O, w.J = a.s.K, w.R = a.s.M, w.splits = p.splits_dw, w.side = p.side_dw, w.cut = p.cut_dw;
    w.part = (float*)at(a.workspace, p.part_dw);
    w.o.out = a.dw, w.o.J = a.s.K, w.o.f32 = a.dw_f32, w.o.accumulate = a.accumulate;
  }
  if (both) {
    GemmPair pair;
    pair.dx = x, pair.dw = w, pair.sums = c;
    return std::is_same_v<T, __bf16> ? launch_gemm_pair_bf16(pair) : launch_gemm_pair_f32(pair);
  }
  if (a.dx) e = launch_product<T>(x);
  if (a.dw && e == hipSuccess) e = launch_product<T>(w);
  return e;
}

}  // namespace

hipError_t launch_column_sums(const ColumnSums& a) {
  hipLaunchKernelGGL(column_sums_kernel, dim3((uint32_t)((a.cols + kSumCols - 1) / kSumCols)),
                     dim3(kSumCols * kSumGroups), 0, a.stream, a);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs& a) {
  return a.s.bf16 ? forward<__bf16>(a) : forward<float>(a);
}

hipError_t launch_linear_bwd(const LinearArgs& a) {
  return a.s.bf16 ? backward<__bf16>(a) : backward<float>(a);
}

}  // namespace ringx
