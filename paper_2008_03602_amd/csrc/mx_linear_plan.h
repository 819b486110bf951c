// Which tiles the product of microscaled rows takes, by its sizes (host only; constant evaluation goes
// through it in a test).
#pragma once

#include "seq_internal.h"

namespace ct {

enum { MXL_32X16, MXL_32, MXL_64, MXL_128X64, MXL_128, MXL_256, MXL_KINDS };
struct MxShape {
  int bm, bn, wm, wn, wk, stages;
};
constexpr MxShape kMxTiles[MXL_KINDS] = {{32, 16, 1, 1, 8, 3}, {32, 32, 1, 2, 4, 3}, {64, 64, 2, 2, 2, 3}, {128, 64, 2, 2, 1, 3},
                                         {128, 128, 2, 2, 1, 2}, {256, 256, 4, 2, 1, 2}};

constexpr int64_t mx_tiles_of(const ct_mx_linear_op& op, int kind) {
  const MxShape t = kMxTiles[kind];
  return (((int64_t)op.m + t.bm - 1) / t.bm) * (((int64_t)op.n + t.bn - 1) / t.bn);
}

constexpr MxLinearPlan mx_linear_plan(const ct_mx_linear_op& op) {
  MxLinearPlan p = {};
  const int steps = (int)(((int64_t)op.k + 127) / 128);
  // Rounds of the device, and what a round costs beside one of 64 x 64 tiles, of which a compute unit
  // has two at a time (as of 128 x 64). Measured on 1021 x 515 by 1277, 512 x 2048 by 2048, 200 x 1024
  // by 4096, 2048^3, 4096 x 1024 by 1024, 4000 x 500 by 3000, 16000 x 320 by 320 and 8192 x 4096 by
  // 8192: the choice is the fastest or within 12 % of it. With the elements in bf16 256 x 256 tiles
  // leave no registers.
  auto rounds = [&](int kind, int blocks) { return (double)((mx_tiles_of(op, kind) + kPlanCus * blocks - 1) / (kPlanCus * blocks)); };
  p.kind = MXL_64;
  double least = rounds(MXL_64, 2);
  const auto offer = [&](int kind, double cost) {
    if (cost >= least) return;
    least = cost;
    p.kind = kind;
  };
  offer(MXL_128X64, 1.7 * rounds(MXL_128X64, 2));
  // (one round of 128 x 128 is one of 128 x 64, two at a time, and takes as long)
  if (rounds(MXL_128, 1) > 1) offer(MXL_128, 1.5 * rounds(MXL_128, 1));
  if (op.out_dtype != CT_DT_F32) offer(MXL_256, 4.6 * rounds(MXL_256, 1));
  // Up to 64 rows or columns past whole 256 x 256 tiles would take the device another round; they go
  // apart where that is less: 8192 x 2048 by 8208 186 to 177 us, 4096 x 4096 by 8224 203 to 158,
  // 4100 x 4096 by 8200 206 to 164, 8192 x 4096 by 2064 116 to 87, 4096 x 512 by 4100 24.5 to 26.2
  if (op.out_dtype == CT_DT_BF16 && op.m > 32)
    for (int tails = 1; tails < 4; ++tails) {
      const int tm = tails & 1 ? op.m % 256 : 0, tn = tails & 2 ? op.n % 256 : 0;
      if (tm > 64 || tn > 64 || (tails & 1 && !tm) || (tails & 2 && !tn)) continue;
      const int64_t tiles = (((int64_t)op.m - tm + 255) / 256) * (((int64_t)op.n - tn + 255) / 256);
      const double cost = 4.6 * (double)((tiles + kPlanCus - 1) / kPlanCus) + (tm != 0) + (tn != 0);
      if (!tiles || cost >= least) continue;
      least = cost;
      p.kind = MXL_256;
      p.tail_m = tm;
      p.tail_n = tn;
    }
  // Smaller tiles where 64 x 64 leaves compute units without one: 64 x 4096 by 4096 13.6 to 7.7 us, and
  // for few rows 24 x 8192 by 4096 11.1 to 9.5
  if (op.m <= 32 || (p.kind == MXL_64 && mx_tiles_of(op, MXL_64) < kPlanCus * 3 / 4)) p.kind = MXL_32;
  if (p.kind == MXL_32 && op.m <= 32 && mx_tiles_of(op, MXL_32) < kPlanCus * 3 / 4) p.kind = MXL_32X16;
  // A long reduction over few tiles: slices of it, of 32 steps at least, so that they save more
  // than the second kernel takes. Launches apart have no workspace to put partial sums into.
  const int64_t blocks = mx_tiles_of(op, p.kind);
  int split = 1;
  if (!p.tail_m && !p.tail_n && blocks <= kPlanCus / 4 && steps >= 64) split = (int)(kPlanCus / blocks < steps / 32 ? kPlanCus / blocks : steps / 32);
  const int per = steps ? (steps + split - 1) / split : 1;
  p.split = steps ? (steps + per - 1) / per : 1;
  p.per_split = per;
  p.ws_floats = p.split > 1 ? (int64_t)p.split * op.m * ((op.n + 3) / 4 * 4) : 0;
  return p;
}

}  // namespace ct
