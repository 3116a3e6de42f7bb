// Host-side launch interface between the C ABI layer (ringx_api.cpp) and the kernel files.
// Arguments arrive here already validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace ringx {

// What the forward does with each chunk's local result (loc_out_r, loc_lse_r).
enum class FwdMode {
  kFused = 0,     // Eq. (5) merge of all R chunks in registers -> out, lse
  kPartials = 1,  // write every chunk's result -> part_out, part_lse
  kStep = 2,      // R = 1: merge the one chunk into the running fp32 acc_out, acc_lse
};

// How the query-stationary bf16 kernels (forward, dQ) cut a launch.  Whole: workgroups of 256
// queries, one per CU, so n of them take ceil(n / 256) rounds, and with few of them, or few in the
// last round, most of the chip is idle.
struct QueryCut {
  int ks = 1;          // key streams: an 8-wave workgroup takes 256 / ks queries, its waves split the
                       // keys ks ways
  bool half = false;   // 4-wave workgroups of 128 queries, three per CU (d = 64)
};
// What a kernel gains beyond rounds that are half empty or emptier.  A kernel with half-size workgroups
// takes them in ragged launches, and in full rounds from n = half_from on, up to half_keys keys;
// one without (half_from = 0) takes two streams in ragged launches, from split_keys[0] keys on up
// to two rounds and from split_keys[1] on up to three.
struct CutRule {
  int64_t half_from, half_keys;
  int64_t split_keys[2];
};
// n = B H ceil(Nq / 256); `keys` that one workgroup visits.  Measured at 8192 keys, two heads (us; one,
// two and four streams, *half-size):
//   n =            96           128          192          288              384              768
//   forward d=64   130 84 96    123 82 92    127 148 136  260 222 195*     259 240 217*     422 458 419*
//   forward d=128  178 127 152  168 130 152  200 222 230  388 338          387 370          679 731
//   dQ d=64        156 94 106   157 103 112  162 180 165  327 275 249*     329 299 282*     566 586
//   dQ d=128       263 157 199  263 181 212  270 311 316  575 485          576 528          963 1043
// and at n = 64, 4096 keys: 66 40 28, 88 54 45, 81 46 34 and 138 81 64.  So: four streams as long
// as one round holds the quarter-size workgroups, two while it holds the half-size ones; where the
// last round is at most half full, half-size workgroups, which end closer together.  In full rounds
// splitting loses, because a tile serves fewer queries, unless three half-size workgroups on a CU
// gain more by covering each other's barriers, first and last tiles:
// the d = 64 forward does up to 16384 keys (n = 1024: 1024 keys 97 -> 85, 4096 301 -> 284, 16384
// 1130 -> 1072; 2% slower at 262144), dQ up to 4096 keys and from three rounds on (1024 keys 118 ->
// 110, n = 768 at 2048 keys 160 -> 153, n = 3072 at 4096 1138 -> 1108; n = 512 197 against 204).
// At d = 128, without half-size workgroups, two streams in a ragged launch have a fixed cost (a
// merge, and a wave's own Q for half as many keys) and pay only where the round they save is long.
// Speed-up over one stream by n and keys (lowest and highest of five n in each range):
//   forward     300         512         1500        4096        8192        16384       32768
//   257 .. 384  0.86 0.89   0.91 0.94   0.96 1.05   1.03 1.09   1.02 1.11   1.06 1.12   1.17 1.24
//   513 .. 640  0.79 0.83   0.85 0.89   0.91 0.94   0.95 0.99   0.98 1.00   0.97 1.09   1.04 1.14
//   769 .. 896  0.74 0.80   0.79 0.82   0.87 0.91   0.91 0.96   0.93 0.97   0.98 1.05   1.01 1.04
//   dQ
//   257 .. 384  1.02 1.06   1.07 1.13   1.07 1.17   1.10 1.11   1.10 1.12   1.12 1.15   1.15 1.26
//   513 .. 640  0.97 0.99   0.99 1.09   1.01 1.03   0.99 1.04   1.01 1.05   1.04 1.13   1.04 1.12
//   769 .. 896  0.96 0.98   0.96 0.98   0.98 1.03   0.96 1.00   0.95 0.99   1.00 1.12   1.00 1.02
inline QueryCut query_cut(int64_t n, int64_t keys, const CutRule& r) {
  QueryCut c;
  const bool ragged = n > 256 && n < 1024 && (n - 1) % 256 < 128;
  if (r.half_from > 0 && (ragged || (n >= r.half_from && keys <= r.half_keys))) c.half = true;
  else if (n <= 64) c.ks = 4;
  else if (n <= 128) c.ks = 2;
  else if (ragged && n <= 768 && keys >= r.split_keys[n <= 512 ? 0 : 1]) c.ks = 2;
  while (c.ks > 1 && keys < 64 * c.ks) c.ks /= 2;
  return c;
}
// half-size forms exist at d = 64 only
inline CutRule fwd_cut_rule(int64_t d) {
  return d == 64 ? CutRule{512, 16384, {0, 0}} : CutRule{0, 0, {2048, 16384}};
}
inline CutRule dq_cut_rule(int64_t d) {
  return d == 64 ? CutRule{768, 4096, {0, 0}} : CutRule{0, 0, {0, 1024}};
}

struct FwdPlan {
  QueryCut cut;
  int64_t rg = 1;   // chunk groups (partials)
};

// n = B H ceil(Nq / 256) as above, R chunks of Nk keys.
// Partials: chunks are independent, so they are spread over workgroups, over as few groups as give
// the shortest launch (480 workgroups, whose two rounds are nearly full, lose 2% to four groups),
// and up to four rounds where one is at most half full (Nq = 2048, 8 chunks of 4096, 16 heads,
// d = 128: 664 us whole, 479 in one round, 453 in four).  A launch's length is its rounds times the
// chunks of the largest group; at d = 128 a chunk costs as much as 320 keys more (its stores) and a
// workgroup 370 (its queries, the first tiles), fitted to the times of whole and grouped launches
// of 130 .. 2000 workgroups, 2 .. 8 chunks of 300 .. 4000 keys.  Without these two, 200 workgroups
// of 8 chunks of 300 keys took eight groups and 1.30 times as long as whole (1000 keys: 1.08).
// d = 64, whose workgroups are half as large in such launches, gained in every grouped launch.
inline FwdPlan fwd_plan(int64_t n, int64_t Nk, int64_t R, int64_t d, bool partials) {
  FwdPlan p;
  if (partials) {
    const double chunk = (double)Nk / (double)R + (d == 128 ? 320 : 0), start = d == 128 ? 370 : 0;
    auto length = [&](int64_t rg) {
      return (double)((n * rg + 255) / 256) * ((double)((R + rg - 1) / rg) * chunk + start);
    };
    for (int64_t rg = 1; rg < R && n * rg < 2048;) {
      rg = 2 * rg < R ? 2 * rg : R;
      if (length(rg) < 0.97 * length(p.rg) || (n <= 128 && n * rg <= 1024)) p.rg = rg;
    }
  }
  p.cut = query_cut(n * p.rg, Nk / p.rg, fwd_cut_rule(d));
  if (partials) {
    // two streams at most, as the launch is split over chunks already (four 128-key chunks of 4
    // heads x 512 queries: 8.9 us four ways, 10.2 two ways, 12.3 whole), and only where a chunk, not
    // just its group, has a tile for each: the streams split one chunk after the other
    if (p.cut.ks > 2) p.cut.ks = 2;
    if (Nk / R < 64 * p.cut.ks) p.cut.ks = 1;
  }
  return p;
}

// dQ from stored dS: the key-stream kernel (32 queries per workgroup, one of them to a CU) for slabs
// that leave half of the CUs or more without a group of 128 queries and the others with one group
// to hide its own loads.  Its speed-up over the 128-query kernel, R = 1, by keys:
//   groups x queries     32    128   256   512   1000  2000  4000  8000  16000
//   32 x 128             1.16  1.20  1.31  1.48  1.63  1.80  1.91  1.98  2.04
//   64 x 128             1.13  1.16  1.27  1.40  1.56  1.66  1.79  1.86  2.11
//   128 x 32             0.86  0.93  1.08  1.30  1.44  1.48  2.24  2.30  2.18
//   128 x 64             0.96  1.00  1.12  1.33  1.33  1.47  2.06  2.18  2.05
//   96 x 128             0.71  0.73  0.76  0.83  0.88  0.94  0.97  0.99  1.29
//   128 x 128            0.70  0.72  0.77  0.82  0.89  0.98  1.33  1.33  1.32
// (100 chunks of 20 keys, 128 x 128: 1.27; 192 groups even, 256 groups 0.89.)  So: as long as its
// workgroups fit one round, for more than 64 groups from 256 keys on; in two rounds only where
// the 128-query kernel walks many tiles.
inline bool dq_ds_streams(int64_t nh, int64_t Nq, int64_t Nk, int64_t R) {
  const int64_t groups = nh * ((Nq + 127) / 128), wgs = nh * ((Nq + 31) / 32);
  const int64_t tiles = R * (((Nk + R - 1) / R + 63) / 64);
  if (groups > 128) return false;
  if (wgs <= 256) return groups <= 64 || Nk >= 256;
  return tiles >= 96;
}

// The row-streaming tokenizer kernel on rows of more than 128 cells: one field row in flight instead of
// eight (then with a row's 256-cell segments in neighbouring waves at k = 2, a whole sweep of rows
// apart otherwise).
struct TokRowsForm {
  bool one_row = false;
};
// Measured (us; a kernel that loads with a branch per row / one row, segments near / one row, far /
// eight rows, near; 4 channels; crops that start on a 16-byte boundary, off one, and on one with
// the field's edge inside; 64^2 x 512 and 640 with 2 channels):
//   k = 2   512^3, patch 2     670 769 720    665 739 690    686 763 727    704 751 735
//           1024^3, ratio 2    761 808 815    751 774 715    767 812 819    789 812 748
//   k = 4   512^3              390 468 437    384 391 395    391 433 438    374 382 391
//           1024^3, ratio 2    380 423 424    486 506 433    384 426 429    495 515 422
//           1024^2 x 1536, r 2 615 686 707    592 628 655    615 684 709    590 629 653
//   k = 8   512^3              343 389 383    360 382 363    343 381 384    332 353 350
//           1024^3             2698 3110 3037 2874 2987 2909 2675 3006 3017 2881 2952 3014
//           1024^3, ratio 2    329 368 366    333 357 359    330 368 368    354 381 357
//           64^2 x 640         33 52 33       33 34 34       33 33 33       9 10 9
//   k = 16  512^3              327 432 364    336 367 352    326 359 363    326 348 351
//           1024^3, ratio 2    313 348 348    314 338 340    316 352 351    360 386 341
//   k = 4   1024^3              3002 3703 3453  3103 3234 3127  3048 3573 3469  3152 3394 3185
//   k = 2   64^2 x 512          5.3 6.5 5.1     5.8 5.7 5.4     -               4.9 5.0 4.9
// Small fields take eight rows: they come from caches, and few waves need the loads in flight.
// Large ones take one row at k = 2, whose waves are short; where a crop narrower than its field
// reads whole segments (k = 4: of rows a multiple of 4 KiB apart); at k = 8 for rows of three
// segments or more that start on a boundary; and at k = 4 for whole rows of the largest fields.
inline TokRowsForm tok_rows_form(int64_t k, int64_t rows, int64_t sx, int64_t W, int64_t x0) {
  TokRowsForm f;
  const int64_t cells = rows * k * k * sx;
  if (cells < (int64_t(1) << 27)) return f;
  const bool crop = sx > 256 && sx % 256 == 0 && sx < W;
  if (k == 2) f.one_row = true;
  if (k == 4) f.one_row = (crop && W % 1024 == 0) || (sx == W && x0 == 0 && cells >= int64_t(1) << 31);
  if (k == 8) f.one_row = crop || (sx > 512 && x0 % 4 == 0 && W % 4 == 0);
  if (k == 16) f.one_row = crop;
  return f;
}

struct FwdArgs {
  const void* q = nullptr;
  const void* k = nullptr;
  const void* v = nullptr;
  void* out = nullptr;          // merged output (fused mode)
  float* lse = nullptr;         // merged lse (fused mode)
  float* part_out = nullptr;    // [R,B,H,Nq,d] (partials mode)
  float* part_lse = nullptr;    // [R,B,H,Nq]   (partials mode)
  float* acc_out = nullptr;     // [B,H,Nq,d] running merged output (step mode)
  float* acc_lse = nullptr;     // [B,H,Nq]   running merged lse (step mode)
  bool first = false;           // step mode: the accumulator holds nothing yet
  int64_t BH = 0, Nq = 0, Nk = 0, d = 0, R = 1;
  int64_t H = 1, G = 1;         // query heads per batch; query heads per K/V head (GQA)
  float scale = 1.f;
  hipStream_t stream = nullptr;
};

// Dropout of the attention probabilities, as its kernels are told of it (dropout.h).
struct Drop {
  const uint64_t* rng = nullptr;   // seed, offset (device memory)
  uint32_t thr = 0;                // a score is dropped iff its random byte is below
  float inv_keep = 1.f;            // 256 / (256 - thr)
  uint32_t q0 = 0;                 // generator's index of the launch's first query
  uint32_t kb0 = 0;                // and of its first 32-key block
  uint32_t splits = 1;             // parts of the sweep (dK/dV: of the queries, dQ: of the keys), each in
                                   // workgroups of its own, with outputs [splits, ...]
};

// Dropout, bf16: the forward's key streams, those of the plain forward, which has half-size workgroups for
// ragged launches at d = 64.  With dropout these would spill the mask's registers, and two streams serve:
// n workgroups whole, in two, four streams at 1024 x 4096 (us): 260 175 147 143, 320 175 147 148, 384 175 151
// 178, 448 176 194 202, 512 183 200 231, 576 263 246 261, 640 263 254 287; whole and in two at 256, 512, 1024,
// 2048 keys: 320 27 28, 36 35, 56 50, 95 82; 576 39 44, 53 56, 82 81, 142 135.
inline int drop_fwd_streams(int64_t BH, int64_t Nq, int64_t Nk, int64_t d) {
  const int64_t n = (Nq + 255) / 256 * BH;
  if (d == 64 && n > 256 && (n - 1) % 256 < 128 && Nk >= (n <= 512 ? 512 : 2048) && n <= 768) return 2;
  return fwd_plan(n, Nk, 1, d, false).cut.ks;
}
// Dropout, bf16: parts of the keys for a sweep of them in w workgroups.  Up to 128 workgroups, as many parts
// of at least 512 keys as one round of 256 workgroups holds, at most 32: parts of 256 keys gain no more than
// their launch costs (2 heads of 128, 200 x 700, launched one by one: 15 us whole, 19 in two parts).
inline int key_parts(int64_t w, int64_t Nk) {
  return w > 128 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({256 / w, Nk / 512, 32}));
}
// The forward, whose parts are merged by Eq. (5) in a launch more.  us, whole -> in parts: 2 heads of
// 64, 1873 queries, 5265 keys (w = 60) 42 -> 27; 4/1 of 64, 1000 x 30000 (64) 181 -> 66; 1 of 64, 1 x 8192 (1)
// 56 -> 24; 2 of 128, 4096 x 4096 (128) 51 -> 45; from w = 129 on it loses (160: 74 -> 81 .. 98).
inline int drop_fwd_split(int64_t BH, int64_t Nq, int64_t Nk, int64_t d) {
  const int ks = drop_fwd_streams(BH, Nq, Nk, d);
  return key_parts((Nq + 256 / ks - 1) / (256 / ks) * BH, Nk);
}
// How the backward with dropout, bf16, is cut: dQ's key streams in a workgroup, and where heads and rows are
// few, parts of the dK/dV sweep over queries and of the dQ sweep over keys, whose results are summed by
// a launch more (split_sum.hip).
struct DropCut {
  int ks = 1;         // a dQ workgroup takes 256 / ks queries
  int kv = 1, q = 1;  // parts of at least 256 query rows (128 of a head, a tile) and of 512 keys
};
// Workgroups of its one launch: dK/dV's, each of 128 keys of a K/V head, and dQ's.
inline int64_t drop_bwd_workgroups(const DropCut& c, int64_t BHkv, int64_t BH, int64_t Nq, int64_t Nk) {
  return (Nk + 127) / 128 * BHkv * c.kv + (Nq + 256 / c.ks - 1) / (256 / c.ks) * BH * c.q;
}
// The cut with the shortest time by this model.  A dK/dV workgroup takes `row` us for every query row that it
// sweeps, a dQ workgroup `key` us for every key of a stream, each 4 besides, where 256 of them run; fewer at
// a time run 0.85 as long (a higher clock).  The launch lasts as long as its whole work does on 256 CUs,
// or as its list of workgroups, dK/dV's first, on CUs that take the next one when they are free.  Parts
// are written and read at 4 TB/s, and their launch takes 4.  Fitted to times like these (us; dQ streams, *
// parts of dK/dV, + of dQ; model in brackets):
//   heads    queries x keys   one          two         four         others
//   16 d64   4096 x 4096      295 (285)    294 (291)
//   12 d64   3000 x 3000      141 (129)    159 (134)   151 (134)    2* one 158 (155)
//   8 d64    2048 x 2048      59 (53)      48 (44)     48 (46)      2* two 69 (65)
//   32/8 d64 1500 x 5003      257 (259)    277 (264)   292 (281)    2* two 290 (293)
//   4/1 d64  1000 x 30000                              301 (266)    4+ 149 (147), 8+ 153 (153), 2* 4+ 159 (166)
//   8 d128   4096 x 4096      278 (271)    243 (236)
//   5 d128   4096 x 4096      166 (152)    196 (163)   187 (176)    2* two 181 (177)
//   3 d128   8192 x 8192      536 (528)    425 (392)   372 (386)    2* one 434 (443)
//   2 d128   4096 x 4096                               118 (124)    2* 80 (83), 3* two 107 (100), 4* 110 (110)
//   8/1 d128 2048 x 8192                               434 (469)    2* 254 (271), 2* two 259 (251)
// dQ's workgroups first is even or slower in all cuts that it picks.
inline DropCut drop_cut(int64_t BHkv, int64_t BH, int64_t Nq, int64_t Nk, int64_t d, bool parts) {
  constexpr int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  const double row = d == 64 ? 0.020 : 0.033;
  const int64_t sweep = Nq * (BH / BHkv), n1 = (Nk + 127) / 128 * BHkv;
  // nk dK/dV workgroups of tk each, then nq dQ workgroups of tq
  auto length = [](int64_t nk, double tk, int64_t nq, double tq) {
    const int64_t full = nk / 256, rest = nk % 256;
    double a = full * tk + tq, b = (full + 1) * tk + tq;   // next ends on the 256 - rest CUs, on the others
    double t = 0;
    for (int64_t done = 0; done < nq;) {
      const bool late = rest > 0 && b <= a;
      t = late ? b : a;
      done += late ? rest : 256 - rest;
      (late ? b : a) += tq;
    }
    return std::max(t, (full + (rest > 0)) * tk);
  };
  DropCut best;
  double best_us = 0;
  for (int kv : kParts) {
    if (kv > 1 && (!parts || n1 >= 1024 || kv > std::min(Nq / 128, sweep / 256))) break;
    const double tk = (double)sweep / kv * row;
    for (int ks = 1; ks <= 4; ks *= 2) {
      const int64_t n2 = (Nq + 256 / ks - 1) / (256 / ks) * BH;
      if (ks > 1 && (Nk < 64 * ks || n2 / ks >= 1024)) break;
      for (int q : kParts) {
        if (q > 1 && (!parts || ks < 4 || n2 > 256 || q > Nk / 512)) break;
        const double key = d == 64 ? (ks == 1 ? 0.0255 : ks == 2 ? 0.026 : 0.029)
                                   : (ks == 1 ? 0.041 : ks == 2 ? 0.043 : 0.055);
        const double tq = (double)Nk / (ks * q) * key;
        double us = (double)(n1 * kv) * (tk + 4) / 256 + (double)(n2 * q) * (tq + 4) / 256;
        us = std::max(us, length(n1 * kv, 0.85 * tk + 4, n2 * q, 0.85 * tq + 4));
        if (kv > 1) us += (double)(kv * BHkv * Nk * d) * 16 / 4e6;
        if (q > 1) us += (double)(q * BH * Nq * d) * 8 / 4e6;
        if (kv > 1 || q > 1) us += 4;
        if (best_us == 0 || us < best_us) best_us = us, best = {ks, kv, q};
      }
    }
  }
  return best;
}

// out = (out +) sum of `splits` parts of 4 n4 floats
struct SplitSum {
  const float* part = nullptr;
  float* out = nullptr;
  int64_t n4 = 0;
  int splits = 1, accumulate = 0;
};
struct SplitSums {
  SplitSum sum[3];
  int count = 0;
};

struct MergeArgs {
  const float* part_out = nullptr;
  const float* part_lse = nullptr;
  void* out = nullptr;
  float* lse = nullptr;
  int64_t R = 1, BH = 0, Nq = 0, d = 0;
  bool out_bf16 = false;
  hipStream_t stream = nullptr;
};

struct BwdArgs {
  const void* q = nullptr;
  const void* k = nullptr;
  const void* v = nullptr;
  const void* out = nullptr;
  const void* dout = nullptr;
  const float* lse = nullptr;
  float* dq = nullptr;
  float* dk = nullptr;
  float* dv = nullptr;
  float* delta = nullptr;       // D_i = dout_i . out_i, [B,H,Nq]
  float* nl = nullptr;          // -lse_i * log2(e), [B,H,Nq] (the exponent's offset, base 2)
  int64_t BH = 0, Nq = 0, Nk = 0, d = 0, R = 1;   // BH = B * H query heads
  int64_t H = 1, G = 1;         // query heads per batch; query heads per K/V head (GQA)
  float scale = 1.f;
  float d_factor = 1.f;         // preprocess: D is stored times this
  bool accumulate_dkv = false;  // dk, dv += instead of =
  bool accumulate_dq = false;   // dq += instead of =
  char* ds = nullptr;           // store mode of the dK/dV kernel: -dS of every score, bf16
  hipStream_t stream = nullptr;
};

// Stored dS (written by the dK/dV kernel in store mode, read by bwd_dq_ds.hip): per query head j,
// 32-key block kb of the padded key axis (chunk r, 128-key tile t, block w: kb = 4 (r tpc + t) + w,
// nkb = 4 R tpc blocks), 128-query group qg and 32-query block qs of the group, one unit of
// kDsUnitBytes.  The query axis runs fastest, so that each wave of the writer, which owns one key
// block and sweeps the queries, writes one contiguous stream.
constexpr int64_t kDsUnitBytes = 2048;
__host__ __device__ inline int64_t ds_unit_offset(int64_t j, int64_t qg, int64_t kb, int64_t qs,
                                                  int64_t nqg, int64_t nkb) {
  return (((j * nkb + kb) * nqg + qg) * 4 + qs) * kDsUnitBytes;
}
// 128-key tiles per chunk (the longest chunk, ceil(Nk / R) keys, rounded up)
__host__ __device__ inline int64_t ds_tiles_per_chunk(int64_t Nk, int64_t R) {
  return ((Nk + R - 1) / R + 127) / 128;
}
// bytes of stored dS for nh query heads
inline int64_t ds_bytes(int64_t nh, int64_t Nq, int64_t Nk, int64_t R) {
  return nh * ((Nq + 127) / 128) * 4 * R * ds_tiles_per_chunk(Nk, R) * 4 * kDsUnitBytes;
}

struct DsArgs {
  const void* ds = nullptr;     // stored -dS of nh query heads
  const void* k = nullptr;      // K of the nh / G K/V heads, [nh / G, Nk, 128] bf16
  float* dq = nullptr;          // [nh, Nq, 128] fp32, overwritten
  int64_t nh = 0, G = 1, Nq = 0, Nk = 0, R = 1, tpc = 1;
  float scale = 1.f;
  hipStream_t stream = nullptr;
};

// One fidelity mode of the multi-fidelity tokenizer (tt_tokenize.hip).
constexpr int kMaxTokFilter = 32;
struct TokWeights {
  float w[kMaxTokFilter];       // normalised 1D Gaussian weights, w[0 .. k-1]
};
struct TokArgs {
  const float* field = nullptr;  // [C, D, H, W] fp32
  void* tokens = nullptr;        // [L, C p^3], fp32 or bf16
  int64_t C = 0, D = 0, H = 0, W = 0, k = 1, p = 1;
  int64_t gz = 0, gy = 0, gx = 0;   // filtered grid: subdomain size / k
  int64_t z0 = 0, y0 = 0, x0 = 0;   // first subdomain cell, in [0, D) x [0, H) x [0, W)
  TokWeights w{};
  bool out_bf16 = false;
  hipStream_t stream = nullptr;
};

// Norm, rotation and layout change between a packed projection and the attention's operands
// (norm_rope.hip).
struct RopeArgs {
  const void* x = nullptr;       // [B, N, (H + 2 Hkv) d], batch and token strides bs, ts (elements)
  int64_t bs = 0, ts = 0;
  void *q = nullptr, *k = nullptr, *v = nullptr;               // forward: outputs
  const float *dq = nullptr, *dk = nullptr, *dv = nullptr;     // backward: inputs
  void* dx = nullptr;            // backward: [B, N, (H + 2 Hkv) d]
  const float *qw = nullptr, *kw = nullptr;                    // [d] or null
  float *dqw = nullptr, *dkw = nullptr;                        // backward: [d] or null
  float* part = nullptr;         // backward: the workgroups' parts of dqw, dkw; null without weights
  const double* freqs = nullptr;
  const int32_t* pos = nullptr;  // [.., N, axes], null: pos0 + n
  int64_t pos_bs = 0, pos0 = 0;
  int64_t B = 0, N = 0;
  int H = 1, Hkv = 1, d = 0;
  int axes = 1, rot[3] = {0, 0, 0};
  float eps = 0.f;
  bool bf16 = false, vec = true; // vec: rows in 16-byte pieces
  hipStream_t stream = nullptr;
};
// lanes that hold a row
inline int rope_lanes(int64_t d, bool bf16) {
  if (bf16) return (int)(d / 8);
  int l = 1;
  while (4 * l < d) l *= 2;
  return l;
}
// Workgroups of 4 waves along tokens and along heads.  A token's heads are split only to fill the chip,
// since every workgroup forms its tokens' angles: up to 1024 workgroups forward and, where each also
// leaves a part of the weights' gradients, about 512 backward.  Measured in bf16 (us; 256, 512, 1024, 2048; 16
// heads of 128, the last 16/4 of 64); fp32, whose kernels take fewer registers (56 to 70 forward against 100),
// follows the same numbers unmeasured:
//              512 tokens             2048                   8192                   2 x 4097
//   forward    7.2 6.6 7.2 9.2        18.9 12.8 11.4 15.2    35.5 35.0 33.0 33.0    18.1 13.5 14.5 17.5
//   backward   12.3 11.6 13.6 16.8    30.6 22.1 22.9 27.0    78.4 78.4 79.6 82.6    30.8 23.1 29.0 30.8
// Backward workgroups take further tokens beyond 2048, so that the parts stay few.
struct RopeGrid {
  int64_t x, y;
};
inline RopeGrid rope_grid(int64_t rows, int heads, int tokens_per_wave, bool bwd) {
  RopeGrid g;
  const int64_t groups = (rows + 4 * tokens_per_wave - 1) / (4 * tokens_per_wave);
  g.y = 1;
  while (g.y < heads && groups * (g.y + 1) <= (bwd ? 640 : 1024)) ++g.y;
  g.x = bwd && groups > 2048 ? 2048 : groups;
  return g;
}

hipError_t launch_fwd_bf16(const FwdArgs& a, FwdMode mode);
hipError_t launch_fwd_f32(const FwdArgs& a, FwdMode mode);
hipError_t launch_lse_merge(const MergeArgs& a);
hipError_t launch_split_sums(const SplitSums& a, hipStream_t stream);
hipError_t launch_bwd_pre(const BwdArgs& a, bool bf16);
hipError_t launch_bwd_dkdv_bf16(const BwdArgs& a);
hipError_t launch_bwd_dkdv_bf16_d64(const BwdArgs& a);   // d = 64 (bwd_bf16_d64.hip)
hipError_t launch_bwd_dq_bf16(const BwdArgs& a);
// d = 64, and d = 128 where the launch is split into key streams (bwd_dq_bf16_d64.hip)
hipError_t launch_bwd_dq_bf16_two_waves(const BwdArgs& a, const QueryCut& c);
hipError_t launch_bwd_dkdv_f32(const BwdArgs& a);
hipError_t launch_bwd_dq_f32(const BwdArgs& a);
hipError_t launch_bwd_f32(const BwdArgs& a);      // both halves of the fp32 backward
hipError_t launch_bwd_dq_ds(const DsArgs& a);   // d = 128, bf16 dS (bwd_dq_ds.hip)

// with dropout (R = 1; fused and step mode; D of the preprocess times 1 - p)
hipError_t launch_fwd_drop_bf16(const FwdArgs& a, FwdMode mode, const Drop& drop);
hipError_t launch_fwd_drop_f32(const FwdArgs& a, FwdMode mode, const Drop& drop);
// dK/dV and dQ, each in its parts, dQ in ks key streams
hipError_t launch_bwd_drop_bf16(const BwdArgs& a, const Drop& drop_kv, const Drop& drop_q, int ks);
hipError_t launch_bwd_drop_f32(const BwdArgs& a, const Drop& drop);

hipError_t launch_norm_rope(const RopeArgs& a, bool bwd);

hipError_t launch_tt_tokenize(const TokArgs& a);

int64_t fwd_bf16_workgroups(int64_t BH, int64_t Nq, int64_t d);

}  // namespace ringx
