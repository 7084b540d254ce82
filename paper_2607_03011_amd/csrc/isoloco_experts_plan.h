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
inline ExpertPlan expert_plan(ExpertProduct p, bool f32, int64_t rows, int64_t experts, int64_t m, int64_t n, int64_t k) {
  const double parts = f32 ? 6 : 1;
  const double depth = p == kDw ? std::max(1.0, (double)rows / experts / kSlab) * parts
                                : (double)std::max<int64_t>(1, (k + kSlab - 1) / kSlab) * parts;
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
      if (q > 1) us += (double)q * (p == kDw ? experts * m : rows) * n * 8 / 3e6 + kJoinUs;
      if (us < best.us) best = {s, q, us};
    }
  }
  return best;
}

inline size_t expert_partial_bytes(const ExpertPlan& p, ExpertProduct product, int64_t rows, int64_t experts, int64_t m,
                                   int64_t n) {
  return p.splits > 1 ? (size_t)p.splits * (product == kDw ? experts * m : rows) * ffn_pad(n) * sizeof(float) : 0;
}

}  // namespace isoloco
