// The tile products of the gated feed-forward block: their kinds, and which tiles and
// splits one takes.  Host arithmetic alone.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace isoloco {

// da and du, and copies of x and the weights, have their columns padded to multiples of
// this (the k values of a slab), da and du their rows too, zeros in the padding: the
// products that sum over a padded extent need no bounds there.
constexpr int kFfnPad = 64;
constexpr int64_t ffn_pad(int64_t v) { return (v + kFfnPad - 1) / kFfnPad * kFfnPad; }

enum FfnMode {
  kForward,  // out[0] = act(a b0^T) (a b1^T)
  kInner,    // out[0] = dh u act'(g), out[1] = dh act(g), padded; in parts if float32
  kSum,      // out[0] = a[0] b[0]^T + a[1] b[1]^T
  kPair      // out[z] = a[z] b[0]^T, z = 0, 1
};

constexpr int kSlab = kFfnPad;

enum ShapeId { kLarge, kMiddle, kSmall, kShapes };
struct ShapeInfo {
  int tm, tn, per_cu;
  float slab_us;  // a slab of the tiles that share a CU
};
constexpr ShapeInfo kShape[kShapes] = {{256, 256, 1, 1.72f}, {192, 256, 1, 1.40f}, {128, 128, 2, 1.05f}};
constexpr int kCus = 256;
constexpr int kMaxSplits = 16;

struct Plan {
  int shape, splits;
  double us;
};

inline int64_t slabs_of(int mode, bool f32, int64_t k) {
  return (k + kSlab - 1) / kSlab * (mode == kSum ? 2 : 1) * (f32 ? 6 : 1);
}
inline int64_t tiles_of(const ShapeInfo& h, int mode, int64_t m, int64_t n) {
  const bool dual = mode == kForward || mode == kInner;
  return ((m + h.tm - 1) / h.tm) * ((n * (dual ? 2 : 1) + h.tn - 1) / h.tn) * (mode == kPair ? 2 : 1);
}
// a round of `slabs`; the splits' sums to memory and back
inline double round_us(const ShapeInfo& h, int64_t slabs) { return (double)slabs * h.slab_us + 4.0; }
inline double sums_us(int mode, int splits, int64_t m, int64_t n) {
  return splits > 1 ? (double)splits * (mode == kSum ? 1 : 2) * m * n * 8 / 3e6 : 0.0;
}
constexpr double kJoinUs = 6.0;

// The tiles and splits that take the least time by the rounds of the launch, the
// slabs of a round and the traffic of the splits' sums.  Both sides measured, us of calls
// in turn on 256-square / 192 x 256 / 128-square tiles: 16384 tokens of 2048 x 5632,
// forward 629 / 665 / 774, dx 635 / 769 / 805, weight gradients 727 / 724 / 887 (352
// tiles of the first are two rounds of 256, the second of them 3/8 full, and cards differ
// in which of the first two is ahead); forward of 2048 tokens, 768 x 2048, 22.4 / 18.9 /
// 17.8.  Splits 1 / 2 / 4 / 8 / 16 of the dx of 512 tokens, 2048 x 5632: 126 / 73 / 45 /
// 44 / 59.
inline Plan plan_of(int mode, bool f32, int64_t m, int64_t n, int64_t k) {
  const int64_t slabs = slabs_of(mode, f32, k);
  Plan best = {kSmall, 1, 1e30};
  for (int s = 0; s < kShapes; ++s) {
    const ShapeInfo& h = kShape[s];
    const int64_t tiles = tiles_of(h, mode, m, n);
    for (int p = 1; p <= kMaxSplits && (p == 1 || p * 4 <= slabs); ++p) {
      const int64_t rounds = (tiles * p + kCus * h.per_cu - 1) / (kCus * h.per_cu);
      const double us =
          rounds * round_us(h, (slabs + p - 1) / p) + sums_us(mode, p, m, n) + (p > 1 ? kJoinUs : 0.0);
      if (us < best.us) best = {s, p, us};
    }
  }
  return best;
}

// kSum of m x n over k with kPair of k x n over m: one launch where that takes less than
// the two apart by the same rule (1.06: of which it leaves out that the first of two
// drains before the second fills the card).  Both sides measured, us of the whole
// gradient, apart / together: bfloat16, 512 tokens of 768 x 2048 42 / 35, 4096 tokens 121
// / 97, 1024 of 2048 x 5632 172 / 155, 4096 of them 543 / 501, 8192 of 1024 x 4096 423 /
// 375; float32, 1000 tokens of 612 x 1637 140 / 122, 2048 of 768 x 2048 292 / 268.  Where
// the rule keeps them apart: 3000 tokens of 1001 x 2777 in float32 729 / 774.
struct GradientsPlan {
  bool together;
  Plan sum, pair;
};
constexpr int kTogether[][2] = {{kSmall, kSmall}, {kLarge, kLarge}, {kLarge, kMiddle}};
inline GradientsPlan plan_gradients(bool f32, int64_t m, int64_t n, int64_t k) {
  GradientsPlan best = {false, plan_of(kSum, f32, m, n, k), plan_of(kPair, f32, k, n, m)};
  if (m == 0) return best;
  double least = 1.06 * (best.sum.us + best.pair.us);
  const int64_t slabs_s = slabs_of(kSum, f32, k), slabs_p = slabs_of(kPair, f32, m);
  for (const auto& shapes : kTogether) {
    const ShapeInfo &hs = kShape[shapes[0]], &hp = kShape[shapes[1]];
    const int64_t tiles_s = tiles_of(hs, kSum, m, n), tiles_p = tiles_of(hp, kPair, k, n), slots = kCus * hs.per_cu;
    for (int p = 1; p <= kMaxSplits && (p == 1 || p * 4 <= slabs_s); ++p) {
      // as many splits of the other as its slabs take no longer with
      const int64_t length = (slabs_s + p - 1) / p;
      for (int64_t more = 0; more < 2; ++more) {
        const int64_t q = std::min<int64_t>(kMaxSplits, (slabs_p + length - 1) / length + more);
        if (q > 1 && q * 4 > slabs_p) continue;
        const double us_s = round_us(hs, length), us_p = round_us(hp, (slabs_p + q - 1) / q);
        const int64_t ns = tiles_s * p, np = tiles_p * q;
        // the workgroups follow each other; the last of them end at different times
        double us = std::max(us_s, us_p);
        if (ns + np > slots) us = std::max(us, (ns * us_s + np * us_p) / slots + 0.5 * us_p);
        us += sums_us(kSum, p, m, n) + sums_us(kPair, (int)q, k, n) + (p > 1 || q > 1 ? kJoinUs : 0.0);
        if (us < least) {
          least = us;
          best = {true, {shapes[0], p, us}, {shapes[1], (int)q, us}};
        }
      }
    }
  }
  return best;
}

inline size_t partial_bytes(const Plan& p, int mode, int64_t m, int64_t n) {
  return p.splits > 1 ? (size_t)p.splits * (mode == kSum ? 1 : 2) * m * ffn_pad(n) * sizeof(float) : 0;
}

}  // namespace isoloco
