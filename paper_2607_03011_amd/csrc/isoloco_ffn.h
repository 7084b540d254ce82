// The products of the gated feed-forward block, shared by its kernel files.
#pragma once
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "isoloco.h"

namespace isoloco {

// act(g) and its derivative
template <int ACT>
__device__ __forceinline__ void activate(float g, float& a, float& da) {
  if constexpr (ACT == ISOLOCO_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else {
    const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * cdf;
    da = cdf + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  }
}

// The same where the result is rounded to bfloat16 after it: the hardware's
// exponential and reciprocal (1 ulp), and for the normal CDF the rational
// approximation 7.1.26 of Abramowitz and Stegun (absolute error 8e-8).  The library
// functions cost a forward pass of 16384 tokens, 2048 x 5632, a tenth of its time.
template <int ACT>
__device__ __forceinline__ void activate_fast(float g, float& a, float& da) {
  constexpr float kLog2e = 1.44269504088896340736f;
  if constexpr (ACT == ISOLOCO_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else {
    const float x = fabsf(g) * 0.70710678118654752f, e = __builtin_amdgcn_exp2f(-kLog2e * x * x);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f),
                             0.254829592f);
    const float tail = 0.5f * p * e;  // Phi(-|g|)
    const float cdf = g < 0.f ? tail : 1.f - tail;
    a = g * cdf;
    da = fmaf(g * 0.39894228040143268f, e, cdf);
  }
}

// An operand of a product: element (row, k) at p + row * rs + k * ks (elements),
// one of the strides 1.
struct Operand {
  const void* p;
  int64_t rs, ks;
};

enum FfnMode {
  kForward,  // out[0] = act(a b0^T) (a b1^T)
  kInner,    // out[0] = dh u act'(g), out[1] = dh act(g)
  kSum,      // out[0] = a[0] b[0]^T + a[1] b[1]^T
  kPair      // out[z] = a[z] b[0]^T, z = 0, 1
};

struct FfnArgs {
  Operand a[2], b[2];
  int64_t m, n, k;
  void* out[2];
  int64_t ld_out;
  const void* dh;
  int64_t ld_dh;
};

// da and du are kept with their rows and columns padded to multiples of this (the
// k values of a slab of the tile kernels), zeros in the padding: the products that
// sum over either need no bounds there.
constexpr int kFfnPad = 64;
__host__ __device__ inline int64_t ffn_pad(int64_t v) { return (v + kFfnPad - 1) / kFfnPad * kFfnPad; }

// The bfloat16 products on tiles: every row of every operand 16-byte aligned, and
// (kForward, kInner) k a multiple of 8, (kSum, kPair) n a multiple of 8 and a as
// kInner left it.
// `partial`: ffn_partial_bytes() of memory for the sums of a product whose k values
// are split over workgroups (kSum and kPair with few tiles).
size_t ffn_partial_bytes(FfnMode mode, int64_t m, int64_t n, int64_t k);
hipError_t launch_ffn_tiles(FfnMode mode, int act, const FfnArgs& g, float* partial, hipStream_t st);

}  // namespace isoloco
