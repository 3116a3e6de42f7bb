// How the tiled matrix products of the linear layer get their operands into LDS (gfx950).
//
// out[i][j] = sum over r of P(i, r) Q(j, r).  A workgroup makes a tile of out; operands go through LDS in steps of
// 128 bytes along r, two buffers filled by direct global->LDS loads: while one step is multiplied, the next one
// is in flight.  An operand that is stored with r along its rows (contiguous) is a tile of W rows; one stored the
// other way (slow: r is the row) a tile of 64 (bf16) or 32 (fp32) rows of W values.  16-byte pieces of a row are
// XOR-swizzled by the row so that the reads of fragments do not meet themselves in a bank: contiguous tiles by
// (row / 2) mod 8 (16 lanes read one piece of 16 rows); slow ones in bf16 by 4 (row mod 4) + (row / 4) mod 4
// (transposed reads: 16 lanes read 32 bytes of 4 rows), in fp32 by 8 ((row / 4) mod 2) (32 lanes read 128 bytes of
// a row, the others those of the fourth row after it).
//
// All loads are buffer loads from the tile's place on: what lies past the tensor's end reads as zero, and
// so do the pieces past R in the last step, whose offsets are moved outside.  Rows of i or j past the
// end repeat the last one (contiguous) or are what follows (slow): they reach only values that are not
// stored.
#pragma once

#include "ringx_device.h"
#include "ringx_kernels.h"

namespace ringx {
namespace {

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

// One operand's way into LDS, 128 bytes of r at a time: a tile of W rows of 128 bytes, or, where r is the row
// (SLOW), of BK rows of W values.
template <class T, bool SLOW, int W, int THREADS>
struct Feed {
  static constexpr int kSize = (int)sizeof(T), E = 16 / kSize, BK = 128 / kSize;   // values of a piece, of a step
  static constexpr int kLoads = W * 128 / (THREADS * 16);
  static constexpr int kRowChunks = SLOW ? W / E : 8;
  static_assert(kLoads * THREADS * 16 == W * 128 && kRowChunks % 8 == 0, "whole rounds of loads");
  static_assert(!SLOW || kRowChunks >= 16, "the swizzle stays in a row");
  static_assert(SLOW || THREADS / kRowChunks % 16 == 0, "rounds keep the swizzle's phase");
  uint32_t off[kLoads];
  int64_t base, left;    // address of the step's first row or column; bytes from it to the tensor's end
  int64_t step, turn;    // bytes to the next step; what is added where a head (or batch) ends
  int in, per;           // steps left in this head (or batch), steps of one (0: there are none)
  int chunk;             // contiguous: the lane's first r of a step / 8

  static __device__ __forceinline__ int swz(int row) {
    if (!SLOW) return (row >> 1) & 7;
    return kSize == 2 ? ((row & 3) << 2) | ((row >> 2) & 3) : (row >> 2 & 1) << 3;
  }

  // Width index w0 and r0 (a multiple of BK) on.  Sizes fit 32 bits, which divisions are made in: with those
  // of 64 bits a workgroup's start took 1400 instructions, 5 us.
  __device__ __forceinline__ void start(const GemmIn& x, uint32_t w0, uint32_t r0, int tid) {
    const uint32_t rows = (uint32_t)x.rows, cols = (uint32_t)x.cols, ld = (uint32_t)x.ld;
    int64_t total = (int64_t)(rows - 1) * ld + cols, at;   // elements; from the tensor's start
    turn = 0, per = 0, in = 0;
    if constexpr (!SLOW) {
      at = (int64_t)w0 * ld + r0;
      step = 128;
    } else {
      at = (int64_t)r0 * ld + w0;
      step = kSize * BK * (int64_t)ld;
    }
    const uint32_t d = (uint32_t)x.d, tokens = (uint32_t)x.tokens;
    uint32_t b0 = 0;
    if (x.heads) {
      cold_path();
      total = (int64_t)rows * cols;
      if constexpr (!SLOW) {
        b0 = w0 / tokens;
        const uint32_t hd = d / BK, s = r0 / BK;
        at = (int64_t)b0 * tokens * cols + (int64_t)(s / hd) * tokens * d + s % hd * BK;
        per = (int)hd, in = (int)(hd - s % hd);
        turn = kSize * ((int64_t)tokens * d - d);
      } else {
        b0 = r0 / tokens;
        const uint32_t t = r0 - b0 * tokens;
        at = (int64_t)b0 * tokens * cols + (int64_t)t * d;
        step = kSize * BK * (int64_t)d;
        per = (int)(tokens / BK), in = (int)((tokens - t) / BK);
        turn = kSize * (int64_t)(cols - d) * tokens;
      }
    }
    base = uniform64(reinterpret_cast<int64_t>(x.p) + kSize * at);
    left = uniform64(kSize * (total - at));
    chunk = 0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const uint32_t slot = u * THREADS + tid;
      const uint32_t row = slot / kRowChunks;
      const uint32_t c = (slot % kRowChunks) ^ swz(row);
      if constexpr (!SLOW) {
        chunk = (int)c;   // the same for every u: rounds are whole multiples of 16 rows
        off[u] = kSize * (min(w0 + row, rows - 1) - w0) * ld + c * 16;
      } else {
        off[u] = kSize * row * ld + c * 16;
      }
    }
    if (x.heads) {
      cold_path();
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const uint32_t slot = u * THREADS + tid;
        const uint32_t row = slot / kRowChunks;
        const uint32_t c = (slot % kRowChunks) ^ swz(row);
        if constexpr (!SLOW) {
          const uint32_t i = min(w0 + row, rows - 1), b = i / tokens;
          off[u] = kSize * ((b - b0) * tokens * cols + (i - b * tokens) * d) + c * 16;
        } else {
          const uint32_t col = min(w0 + c * E, cols - E);
          const uint32_t h = col / d;
          off[u] = kSize * (h * tokens * d + (col - h * d) + row * d);
        }
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
    inside = SLOW || chunk * E < rest;
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

// Tile t of a product: tiles in groups of 4 along i, so that those at work on one XCD share operands.
__device__ __forceinline__ void place(uint32_t t, uint32_t ti, uint32_t tj, uint32_t& i, uint32_t& j) {
  constexpr uint32_t kGroup = 4;
  const uint32_t g0 = t / (kGroup * tj) * kGroup, gn = min(kGroup, ti - g0);
  t -= g0 * tj;
  i = g0 + t % gn, j = t / gn;
}

}  // namespace
}  // namespace ringx
