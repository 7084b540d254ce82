// Which tiles and splits a product grouped by expert takes.  Host arithmetic alone.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "isoloco_ffn_plan.h"

namespace isoloco {

enum ExpertProduct {
  kOut,  // out[r] = a[r] b[e]^T
  kDx,   // out[r] = a[r] b[e]
  kDw    // out[e] = sum over its rows of a[r]^T b[r]
};

struct ExpertPlan {
  int shape, splits;
  double us;
};

// The experts' sizes are not known here: as many tiles as even ones would have, and half a
// tile more for each.
inline double expert_tiles(const ShapeInfo& h, ExpertProduct p, int64_t rows, int64_t experts, int64_t m, int64_t n) {
  const double tiles_n = (double)((n + h.tn - 1) / h.tn);
  if (p == kDw) return (double)experts * ((m + h.tm - 1) / h.tm) * tiles_n;
  const int64_t groups = std::min(experts, rows);
  const double even = (double)rows / std::max<int64_t>(groups, 1);
  return groups * std::max(1.0, even / h.tm + 0.5) * tiles_n;
}

// The tiles and splits that take the least time by the rounds of the workgroups, as plan_of does
// it.  dw's tiles are as deep as their experts have rows: the workgroups follow each other
// there, and an expert of twice the mean is expected (by whole rounds alone 47 where the
// 128-square tiles take 35.5 us: 4096 rows of 8 experts of 2048 x 768).  Both sides measured, us
// on 256-square / 192 x 256 / 128-square tiles, uneven experts in bfloat16:
//   4096 rows, 8 experts of 2048 x 768     out 25.6 / 21.9 / 28.0   dx 46.4 / 39.8 / 31.1   dw 47.4 / 43.3 / 35.5
//   16384 rows, 8 experts of 1408 x 2048   out 106 / 122 / 107      dx 116 / 97.4 / 115     dw 140 / 154 / 129
//   32768 rows, 64 experts of 512 x 1024   out 56.0 / 48.6 / 53.1   dx 57.5 / 58.6 / 56.6   dw 60.9 / 66.4 / 61.0
// and in 1 / 2 / 3 / 6 splits on 128-square ones: dx of 1400 rows, 5 experts of 1637 x 612 in
// float32 142 / 85 / 70 / 54.
inline double expert_depth(ExpertProduct p, bool f32, int64_t rows, int64_t experts, int64_t k) {
  const double parts = f32 ? 6 : 1;
  return p == kDw ? std::max(1.0, (double)rows / experts / kSlab) * parts
                  : (double)std::max<int64_t>(1, (k + kSlab - 1) / kSlab) * parts;
}
inline double expert_sums_us(ExpertProduct p, int splits, int64_t rows, int64_t experts, int64_t m, int64_t n) {
  return splits > 1 ? (double)splits * (p == kDw ? experts * m : rows) * n * 8 / 3e6 : 0.0;
}
inline ExpertPlan expert_plan(ExpertProduct p, bool f32, int64_t rows, int64_t experts, int64_t m, int64_t n, int64_t k) {
  const double depth = expert_depth(p, f32, rows, experts, k);
  ExpertPlan best = {kSmall, 1, 1e30};
  for (int s = 0; s < kShapes; ++s) {
    if (p == kDw && s == kMiddle) continue;  // (never the least of the three there)
    const ShapeInfo& h = kShape[s];
    const double tiles = expert_tiles(h, p, rows, experts, m, n), slots = kCus * h.per_cu;
    for (int q = 1; q <= kMaxSplits && (q == 1 || q * 4 <= depth); ++q) {
      const double one = depth / q * h.slab_us + 4.0;
      double us;
      if (p == kDw) us = std::max(tiles * q / slots * one, 2 * one - 4.0) + 0.5 * one;
      else us = (double)(int64_t)(std::max(1.0, tiles * q / slots) + 0.999) * one;
      us += expert_sums_us(p, q, rows, experts, m, n) + (q > 1 ? kJoinUs : 0.0);
      if (us < best.us) best = {s, q, us};
    }
  }
  return best;
}

// Both gradients of rows of dim and cols: one launch, whose workgroups take dw's tiles and then
// dx's, where that takes less than the two apart by the same rule (float32: clearly less, its
// splits and 192 x 256 tiles being lost there).  Both sides measured, us of both, apart /
// together: bfloat16, 1024 rows of 8 experts of 2048 x 768 36.4 / 30.7, 4096 rows 66.2 / 59.3, 16384
// of 1408 x 2048 238 / 221, 32768 of 64 experts of 512 x 1024 131 / 115; float32, 1400 rows of 5 of
// 1637 x 612 107 / 99.5; where the rule keeps them apart, 4096 rows of 8 of 2048 x 768 275 / 308.
struct ExpertGradients {
  bool together;
  ExpertPlan dx, dw;
};
inline ExpertGradients expert_plan_gradients(bool f32, int64_t rows, int64_t experts, int64_t dim, int64_t cols) {
  ExpertGradients best = {false, expert_plan(kDx, f32, rows, experts, 0, dim, cols),
                          expert_plan(kDw, f32, rows, experts, cols, dim, 0)};
  if (rows == 0) return best;
  double least = (f32 ? 0.92 : 1.0) * (best.dx.us + best.dw.us);
  const double depth_x = expert_depth(kDx, f32, rows, experts, cols), depth_w = expert_depth(kDw, f32, rows, experts, 0);
  for (const int s : {(int)kLarge, (int)kSmall}) {
    const ShapeInfo& h = kShape[s];
    const double tiles_x = expert_tiles(h, kDx, rows, experts, 0, dim), slots = kCus * h.per_cu;
    const double tiles_w = expert_tiles(h, kDw, rows, experts, cols, dim);
    for (int q = 1; q <= kMaxSplits && (q == 1 || q * 4 <= depth_x); ++q)
      for (int r = 1; r <= kMaxSplits && (r == 1 || r * 4 <= depth_w); ++r) {
        const double one_x = depth_x / q * h.slab_us + 4.0, one_w = depth_w / r * h.slab_us + 4.0;
        double us = std::max((tiles_x * q * one_x + tiles_w * r * one_w) / slots, std::max(one_x, 2 * one_w - 4.0)) +
                    0.5 * std::max(one_x, one_w);
        us += expert_sums_us(kDx, q, rows, experts, 0, dim) + expert_sums_us(kDw, r, rows, experts, cols, dim) +
              (q > 1 || r > 1 ? kJoinUs : 0.0);
        if (us < least) {
          least = us;
          best = {true, {s, q, us}, {s, r, us}};
        }
      }
  }
  return best;
}

inline size_t expert_partial_bytes(const ExpertPlan& p, ExpertProduct product, int64_t rows, int64_t experts, int64_t m,
                                   int64_t n) {
  return p.splits > 1 ? (size_t)p.splits * (product == kDw ? experts * m : rows) * ffn_pad(n) * sizeof(float) : 0;
}

}  // namespace isoloco
