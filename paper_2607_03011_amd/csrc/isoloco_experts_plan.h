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

inline ExpertPlan expert_plan(ExpertProduct p, bool f32, int64_t rows, int64_t experts, int64_t m, int64_t n, int64_t k) {
  const int64_t depth = p == kDw ? (rows + experts - 1) / experts : k;
  const int64_t slabs = std::max<int64_t>(1, (depth + kSlab - 1) / kSlab) * (f32 ? 6 : 1);
  ExpertPlan best = {kSmall, 1, 1e30};
  for (int s = 0; s < kShapes; ++s) {
    const ShapeInfo& h = kShape[s];
    const double tiles = expert_tiles(h, p, rows, experts, m, n);
    for (int q = 1; q <= kMaxSplits && (q == 1 || q * 4 <= slabs); ++q) {
      const double rounds = std::max(1.0, tiles * q / (kCus * h.per_cu));
      const double whole = (double)(int64_t)(rounds + 0.999);
      const double us = whole * round_us(h, (slabs + q - 1) / q) +
                        (q > 1 ? (double)q * (p == kDw ? experts * m : rows) * n * 8 / 3e6 + kJoinUs : 0.0);
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
