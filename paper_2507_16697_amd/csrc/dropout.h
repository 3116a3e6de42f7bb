// Dropout of attention probabilities by a counter-based generator: the mask of a score is a function
// of its place and of the generator's state (seed, offset), so it is never stored: the backward, a
// ring step and a launch that is cut another way form the same bits again.
//
// Generator: Philox4x32 (J. K. Salmon, M. A. Moraes, R. O. Dror, D. E. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC'11) with 7 rounds, the fewest that pass the paper's whole test
// battery.  Key: the seed.  Counter: (16-key group, query, query head of B * H, offset mod 2^32).
// A group is half of a 32-key block: group 2 J + h holds keys 32 J + 8 m + 4 h + e, m, e < 4, and
// byte e of result word m is the score's.  These are the 16 keys of a 32 x 32 score tile that one
// lane holds for its query, so that in the query-stationary kernels a lane's 16 scores take one
// generator call and no exchange.  A score is kept iff its byte is at least thr = round(256 p), so
// the rate is a multiple of 1/256: a byte per score makes the generator a quarter of the vector work
// of a score; 16 bits would double that.
#pragma once

#include "ringx_device.h"
#include "ringx_kernels.h"

#include <type_traits>

namespace ringx {

// The argument of kernels without dropout: Drop's fields, as constants.
struct NoDrop {
  static constexpr const uint64_t* rng = nullptr;
  static constexpr uint32_t thr = 0, q0 = 0, kb0 = 0, splits = 1;
  static constexpr float inv_keep = 1.f;
};

template <class T>
constexpr bool kHasDrop = !std::is_same_v<T, NoDrop>;

// The attention kernels stand in headers and are compiled twice, by a source file without dropout and by
// one with it.  The latter defines RINGX_DROPOUT and so gives them this argument and names of their own; the
// two kernels of the bf16 backward become functions, since with dropout one kernel runs both.
namespace {
#ifdef RINGX_DROPOUT
using DROP = Drop;
#define RINGX_KERNEL(name) name##_drop_kernel
#else
using DROP = NoDrop;
#define RINGX_KERNEL(name) name##_kernel
#endif
}  // namespace

// The generator's state as the kernels hold it (wave-uniform).
struct DropKey {
  uint32_t k0 = 0, k1 = 0, off = 0;
  __device__ __forceinline__ explicit DropKey(const uint64_t* rng) {
    if (!rng) return;
    k0 = __builtin_amdgcn_readfirstlane((uint32_t)rng[0]);
    k1 = __builtin_amdgcn_readfirstlane((uint32_t)(rng[0] >> 32));
    off = __builtin_amdgcn_readfirstlane((uint32_t)rng[1]);
  }
};

// a ^ b ^ c in one instruction (the truth table of three inputs)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return (uint32_t)__builtin_amdgcn_bitop3_b32((int)a, (int)b, (int)c, 0x96);
}

__device__ __forceinline__ u32x4 drop_bytes(uint32_t group, uint32_t query, uint32_t head,
                                            const DropKey& key) {
  uint32_t c0 = group, c1 = query, c2 = head, c3 = key.off, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = xor3((uint32_t)(b >> 32), c1, k0);
    c1 = (uint32_t)b;
    c2 = xor3((uint32_t)(a >> 32), c3, k1);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// Word m of four.
__device__ __forceinline__ uint32_t drop_word(const u32x4& w, uint32_t m) {
  const uint32_t lo = m & 1 ? w[1] : w[0], hi = m & 1 ? w[3] : w[2];
  return m & 2 ? hi : lo;
}

// Bit 7 of every byte: whether the byte is at least thr, the carry of adding 256 - thr, which the
// average of four bytes at once, (a + b + 1) / 2, leaves there.  fill = 255 - thr in every byte.
__device__ __forceinline__ u32x4 drop_flags(const u32x4& w, uint32_t fill) {
  u32x4 f;
#pragma unroll
  for (int m = 0; m < 4; ++m) f[m] = __builtin_amdgcn_lerp(w[m], fill, 0x01010101u);
  return f;
}
// The mask of scores i, i + 1 (i even) for their bf16 pair: all ones in the half of one that is kept.
// The byte permute copies sign bits, of odd bytes only, so the even ones come from a shifted copy.
__device__ __forceinline__ uint32_t drop_pair(const u32x4& f, int i) {
  return __builtin_amdgcn_perm(f[i >> 2], f[i >> 2] << 8, i & 2 ? 0x0B0B0909u : 0x0A0A0808u);
}
// 1 where score i is kept, else 0, from its byte: the byte less thr - 1, clamped to [0, 1].  For the
// kernels that need a mask of fp32 values: a conversion, and a subtraction that runs at the rate of
// fp32 arithmetic, twice that of integer instructions, like the multiply-add and the multiply that take
// it (all-ones words and bit selects instead: 2% slower; lane masks do not fit the scalar registers).
__device__ __forceinline__ float drop_weight(const u32x4& w, int i, float edge) {
  const float b = (float)((w[i >> 2] >> (8 * (i & 3))) & 255u);
  return __builtin_amdgcn_fmed3f(b - edge, 0.f, 1.f);
}

}  // namespace ringx
