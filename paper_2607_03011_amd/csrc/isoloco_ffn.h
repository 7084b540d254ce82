// The products of the gated feed-forward block, shared by its kernel files.
#pragma once
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "isoloco.h"
#include "isoloco_ffn_plan.h"

namespace isoloco {

constexpr float kFfnLog2e = 1.44269504088896340736f;

// act(g) and its derivative.  EXACT: to float32's last bits, for float32 results.
// Otherwise for results that are rounded to bfloat16: the hardware's exponential and
// reciprocal (1 ulp), and for the normal CDF the rational approximation 7.1.26 of
// Abramowitz and Stegun (absolute error 8e-8).  (The library functions made a forward
// pass of 16384 tokens, 2048 x 5632, a tenth longer.)
template <int ACT, bool EXACT>
__device__ __forceinline__ void activate(float g, float& a, float& da) {
  if constexpr (ACT == ISOLOCO_ACT_SILU) {
    const float s = EXACT ? 1.f / (1.f + expf(-g)) : __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kFfnLog2e * g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else if constexpr (EXACT) {
    const float cdf = 0.5f * erfcf(-0.70710678118654752f * g);
    a = g * cdf;
    da = cdf + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  } else {
    const float x = fabsf(g) * 0.70710678118654752f, e = __builtin_amdgcn_exp2f(-kFfnLog2e * x * x);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f),
                             0.254829592f);
    const float tail = 0.5f * p * e;  // Phi(-|g|)
    const float cdf = g < 0.f ? tail : 1.f - tail;
    a = g * cdf;
    da = fmaf(g * 0.39894228040143268f, e, cdf);
  }
}

// The operands of the tile products are bfloat16 matrices: the caller's, a copy with
// padded rows, or (float32) three parts each, x = p0 + p1 + p2 with p0 = bf16(x), p1 =
// bf16(x - p0), p2 = bf16(x - p0 - p1), of which the six products of order 2^-16 and
// above are summed: about float32 accuracy.
constexpr int kFfnParts = 3;

// The tile products.  Operands: rows of ld elements (multiples of 8, at most 2^22),
// 16-byte aligned, parts part_a (part_b) elements apart.
//   kForward, kInner  a: m rows of k, b: n rows of k (k a multiple of 8)
//   kSum              a: m rows of k (as kInner left them), b: k rows of cols_b
//   kPair             a: k rows of m (as kInner left them), b: k rows of cols_b
struct FfnArgs {
  const uint16_t *a[2], *b[2];
  int64_t ld_a, ld_b, part_a, part_b;
  int64_t m, n, k;
  int64_t cols_b;  // columns of b: a multiple of 8, at least n
  void* out[2];
  int64_t ld_out, part_out;
  const void* dh;
  int64_t ld_dh;
  float* partial;  // ..._partial_bytes() for the sums of a product whose k values are split over workgroups
};

// kForward and kInner of m x n over k
size_t ffn_projections_partial_bytes(FfnMode mode, bool f32, int64_t m, int64_t n, int64_t k);
hipError_t launch_ffn_projections(FfnMode mode, int act, bool f32, const FfnArgs& g, hipStream_t st);

// kSum of m x n over k and kPair of k x n over m, either of which may be NULL; their
// `partial` is the same.
size_t ffn_gradients_partial_bytes(bool f32, int64_t m, int64_t n, int64_t k);
hipError_t launch_ffn_gradients(bool f32, const FfnArgs* sum, const FfnArgs* pair, hipStream_t st);

}  // namespace isoloco
