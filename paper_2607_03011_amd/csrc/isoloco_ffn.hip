// The gated feed-forward block: both projections, the activation and the product.
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u                      (x: tokens x dim, W: hidden x dim)
//   da = dh u act'(g),  du = dh act(g)
//   dx = da Wg + du Wu,  dWg = da^T x,  dWu = du^T x
//
// g and u stay in registers: the forward pass writes h only, and the backward pass
// forms them again (4 of its 12 tokens x dim x hidden flops) rather than keep two
// arrays of tokens x hidden between the passes.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_ffn.h"

namespace isoloco {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTile = 64, kStep = 32, kThreads = 256;

// A tile of 64 rows x 32 k in LDS, zeros past the operand's end.
template <typename T>
struct Tile {
  // the padding spreads a column's rows over the banks and keeps bfloat16 rows 16-byte aligned
  static constexpr int kPitch = sizeof(T) == 2 ? kStep + 8 : kStep + 1;
  T v[kTile * kPitch];
  __device__ __forceinline__ void load(const Operand& o, int64_t row0, int64_t rows, int64_t k0, int64_t ks) {
    const T* p = static_cast<const T*>(o.p);
    if (o.ks == 1) {
      const int r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 8;
      const T* at = p + (row0 + r) * o.rs + k0 + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[r * kPitch + c + e] = row0 + r < rows && k0 + c + e < ks ? at[e] : (T)0.f;
    } else {
      const int c = threadIdx.x >> 3, r = (threadIdx.x & 7) * 8;
      const T* at = p + (k0 + c) * o.ks + row0 + r;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[(r + e) * kPitch + c] = row0 + r + e < rows && k0 + c < ks ? at[e] : (T)0.f;
    }
  }
};

template <typename T>
__device__ __forceinline__ void multiply(floatx16& acc, const Tile<T>& a, const Tile<T>& b, int i0, int j0) {
  const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
  const T* pa = a.v + (i0 + row) * Tile<T>::kPitch;
  const T* pb = b.v + (j0 + row) * Tile<T>::kPitch;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < kStep; k += 16)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(pa + k + 8 * half),
                                                    *reinterpret_cast<const bf16x8_t*>(pb + k + 8 * half), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < kStep; k += 2)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(pa[k + half], pb[k + half], acc, 0, 0, 0);
  }
}

// Any sizes, strides and alignments: 64 x 64 outputs per workgroup, 32 x 32 per wave.
template <typename T, int MODE, int ACT>
__global__ void __launch_bounds__(kThreads) ffn_any_kernel(FfnArgs g) {
  constexpr bool DUAL = MODE == kForward || MODE == kInner;
  __shared__ Tile<T> sa, sb[DUAL ? 2 : 1];
  const int64_t row0 = (int64_t)blockIdx.y * kTile, col0 = (int64_t)blockIdx.x * kTile;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i0 = (wave >> 1) * 32, j0 = (wave & 1) * 32;
  floatx16 acc[DUAL ? 2 : 1] = {};
  for (int part = 0; part < (MODE == kSum ? 2 : 1); ++part) {
    const Operand& a = MODE == kPair ? g.a[blockIdx.z] : g.a[part];
    for (int64_t k0 = 0; k0 < g.k; k0 += kStep) {
      __syncthreads();
      sa.load(a, row0, g.m, k0, g.k);
      sb[0].load(g.b[part], col0, g.n, k0, g.k);
      if constexpr (DUAL) sb[1].load(g.b[1], col0, g.n, k0, g.k);
      __syncthreads();
      multiply(acc[0], sa, sb[0], i0, j0);
      if constexpr (DUAL) multiply(acc[1], sa, sb[1], i0, j0);
    }
  }
  const int64_t j = col0 + j0 + (lane & 31);
  if (j >= g.n) return;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int64_t i = row0 + i0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
    if (i >= g.m) continue;
    T* out = static_cast<T*>(g.out[MODE == kPair ? blockIdx.z : 0]) + i * g.ld_out + j;
    if constexpr (DUAL) {
      float a, da;
      activate<ACT>(acc[0][e], a, da);
      if constexpr (MODE == kForward) {
        *out = (T)(a * acc[1][e]);
      } else {
        const float dh = (float)static_cast<const T*>(g.dh)[i * g.ld_dh + j];
        *out = (T)(dh * acc[1][e] * da);
        static_cast<T*>(g.out[1])[i * g.ld_out + j] = (T)(dh * a);
      }
    } else {
      *out = (T)acc[0][e];
    }
  }
}

template <typename T, int MODE, int ACT>
hipError_t launch_any(const FfnArgs& g, hipStream_t st) {
  if (g.m == 0 || g.n == 0) return hipSuccess;
  const dim3 grid((unsigned)((g.n + kTile - 1) / kTile), (unsigned)((g.m + kTile - 1) / kTile), MODE == kPair ? 2 : 1);
  hipLaunchKernelGGL((ffn_any_kernel<T, MODE, ACT>), grid, dim3(kThreads), 0, st, g);
  return hipGetLastError();
}

struct FfnShape {
  int64_t tokens, dim, hidden;
  int32_t dtype, act;
};

// The backward workspace: da, du, and the sums of a split product.
size_t inner_bytes(const FfnShape& s) {
  return 2 * (size_t)ffn_pad(s.tokens) * (size_t)ffn_pad(s.hidden) * dtype_bytes(s.dtype);
}
size_t ffn_workspace(const FfnShape& s, bool backward) {
  if (!backward) return 0;
  size_t partial = 0;
  if (s.dtype == ISOLOCO_BF16)
    partial = std::max(ffn_partial_bytes(kSum, s.tokens, s.dim, s.hidden),
                       ffn_partial_bytes(kPair, s.hidden, s.dim, s.tokens));
  return inner_bytes(s) + partial;
}

// the tile kernels load whole 16-byte pieces of rows, at offsets of 32 bits from a tile's first
bool tile_rows(const void* p, int64_t ld) { return aligned_to(p, 16) && (ld & 7) == 0 && ld <= (1 << 20); }

template <typename T>
bool on_tiles(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w) {
  return sizeof(T) == 2 && (s.dim & 7) == 0 && tile_rows(x, ld_x) && tile_rows(wg, ld_w) && tile_rows(wu, ld_w);
}

template <typename T, int ACT>
hipError_t run_forward(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w,
                       void* out, int64_t ld_out, hipStream_t st) {
  FfnArgs g = {};
  g.a[0] = {x, ld_x, 1};
  g.b[0] = {wg, ld_w, 1};
  g.b[1] = {wu, ld_w, 1};
  g.m = s.tokens;
  g.n = s.hidden;
  g.k = s.dim;
  g.out[0] = out;
  g.ld_out = ld_out;
  if (on_tiles<T>(s, x, ld_x, wg, wu, ld_w)) return launch_ffn_tiles(kForward, ACT, g, nullptr, st);
  return launch_any<T, kForward, ACT>(g, st);
}

template <typename T, int ACT>
hipError_t run_backward(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w,
                        const void* dout, int64_t ld_dout, void* dx, int64_t ld_dx, void* dwg, void* dwu,
                        int64_t ld_dw, void* ws, hipStream_t st) {
  const int64_t ld = ffn_pad(s.hidden);
  T* da = static_cast<T*>(ws);
  T* du = da + ffn_pad(s.tokens) * ld;
  float* partial = reinterpret_cast<float*>(static_cast<char*>(ws) + inner_bytes(s));
  const bool tiles = on_tiles<T>(s, x, ld_x, wg, wu, ld_w);
  FfnArgs g = {};
  g.a[0] = {x, ld_x, 1};
  g.b[0] = {wg, ld_w, 1};
  g.b[1] = {wu, ld_w, 1};
  g.m = s.tokens;
  g.n = s.hidden;
  g.k = s.dim;
  g.out[0] = da;
  g.out[1] = du;
  g.ld_out = ld;
  g.dh = dout;
  g.ld_dh = ld_dout;
  hipError_t e = tiles ? launch_ffn_tiles(kInner, ACT, g, partial, st) : launch_any<T, kInner, ACT>(g, st);
  if (e == hipSuccess && dx) {
    g = {};
    g.a[0] = {da, ld, 1};
    g.a[1] = {du, ld, 1};
    g.b[0] = {wg, 1, ld_w};
    g.b[1] = {wu, 1, ld_w};
    g.m = s.tokens;
    g.n = s.dim;
    g.k = s.hidden;
    g.out[0] = dx;
    g.ld_out = ld_dx;
    e = tiles ? launch_ffn_tiles(kSum, ACT, g, partial, st) : launch_any<T, kSum, ACT>(g, st);
  }
  if (e == hipSuccess && dwg) {
    g = {};
    g.a[0] = {da, 1, ld};
    g.a[1] = {du, 1, ld};
    g.b[0] = {x, 1, ld_x};
    g.m = s.hidden;
    g.n = s.dim;
    g.k = s.tokens;
    g.out[0] = dwg;
    g.out[1] = dwu;
    g.ld_out = ld_dw;
    e = tiles ? launch_ffn_tiles(kPair, ACT, g, partial, st) : launch_any<T, kPair, ACT>(g, st);
  }
  return e;
}

isoloco_status check_shape(const FfnShape& s) {
  // the tiles of a launch are counted in 32 bits, those of its rows in 16
  constexpr int64_t most = (int64_t)65535 * kTile;
  if (s.tokens < 0 || s.tokens > most || s.dim < 1 || s.dim > most || s.hidden < 1 || s.hidden > most)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld tokens, dim %lld, hidden %lld", (long long)s.tokens, (long long)s.dim,
                (long long)s.hidden);
  if (!is_dtype(s.dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", s.dtype);
  if (s.act != ISOLOCO_ACT_SILU && s.act != ISOLOCO_ACT_GELU) return fail(ISOLOCO_ERR_INVALID_ARG, "activation %d", s.act);
  return ISOLOCO_OK;
}

struct Range {
  const char* name;
  const void* p;
  size_t bytes;
};

// every output (and the workspace) apart from every input and from each other
template <int NO, int NI>
isoloco_status check_apart(const Range (&out)[NO], const Range (&in)[NI]) {
  for (int i = 0; i < NO; ++i) {
    for (const Range& r : in)
      if (out[i].p && ranges_overlap(out[i].p, out[i].bytes, r.p, r.bytes))
        return fail(ISOLOCO_ERR_ALIAS, "%s overlaps %s", out[i].name, r.name);
    for (int j = 0; j < i; ++j)
      if (out[i].p && out[j].p && ranges_overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return fail(ISOLOCO_ERR_ALIAS, "%s overlaps %s", out[i].name, out[j].name);
  }
  return ISOLOCO_OK;
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

#define BY_TYPES(RUN, ...)                                                                              \
  (dtype == ISOLOCO_F32 ? (act == ISOLOCO_ACT_SILU ? RUN<float, ISOLOCO_ACT_SILU>(__VA_ARGS__)          \
                                                   : RUN<float, ISOLOCO_ACT_GELU>(__VA_ARGS__))         \
                        : (act == ISOLOCO_ACT_SILU ? RUN<__bf16, ISOLOCO_ACT_SILU>(__VA_ARGS__)         \
                                                   : RUN<__bf16, ISOLOCO_ACT_GELU>(__VA_ARGS__)))

extern "C" {

isoloco_status isoloco_gated_ffn_workspace_size(int64_t tokens, int64_t dim, int64_t hidden, int32_t dtype,
                                                int32_t backward, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  const FfnShape s = {tokens, dim, hidden, dtype, ISOLOCO_ACT_SILU};
  ISOLOCO_TRY(check_shape(s));
  *bytes = ffn_workspace(s, backward != 0);
  return ISOLOCO_OK;
}

isoloco_status isoloco_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w,
                                 int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden, int32_t act, void* out,
                                 int64_t ld_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const FfnShape s = {tokens, dim, hidden, dtype, act};
  ISOLOCO_TRY(check_shape(s));
  if (tokens == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), need = ffn_workspace(s, false);
  ISOLOCO_TRY(check_matrix("x", x, tokens, dim, ld_x, e));
  ISOLOCO_TRY(check_matrix("w_gate", w_gate, hidden, dim, ld_w, e));
  ISOLOCO_TRY(check_matrix("w_up", w_up, hidden, dim, ld_w, e));
  ISOLOCO_TRY(check_matrix("out", out, tokens, hidden, ld_out, e));
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const size_t wb = matrix_bytes(hidden, dim, ld_w, e);
  const Range outs[] = {{"out", out, matrix_bytes(tokens, hidden, ld_out, e)}, {"the workspace", workspace, need}};
  const Range ins[] = {{"x", x, matrix_bytes(tokens, dim, ld_x, e)}, {"w_gate", w_gate, wb}, {"w_up", w_up, wb}};
  ISOLOCO_TRY(check_apart(outs, ins));
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const hipError_t r = BY_TYPES(run_forward, s, x, ld_x, w_gate, w_up, ld_w, out, ld_out, st);
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gated feed-forward block");
}

isoloco_status isoloco_gated_ffn_backward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up,
                                          int64_t ld_w, int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden,
                                          int32_t act, const void* dout, int64_t ld_dout, void* dx, int64_t ld_dx,
                                          void* dw_gate, void* dw_up, int64_t ld_dw, void* workspace,
                                          size_t workspace_bytes, void* hip_stream) {
  const FfnShape s = {tokens, dim, hidden, dtype, act};
  ISOLOCO_TRY(check_shape(s));
  const size_t e = dtype_bytes(dtype), need = ffn_workspace(s, true);
  if ((dw_gate != nullptr) != (dw_up != nullptr))
    return fail(ISOLOCO_ERR_INVALID_ARG, "dw_gate and dw_up go together");
  ISOLOCO_TRY(check_matrix("x", x, tokens, dim, ld_x, e));
  ISOLOCO_TRY(check_matrix("w_gate", w_gate, hidden, dim, ld_w, e));
  ISOLOCO_TRY(check_matrix("w_up", w_up, hidden, dim, ld_w, e));
  ISOLOCO_TRY(check_matrix("dout", dout, tokens, hidden, ld_dout, e));
  if (dx) ISOLOCO_TRY(check_matrix("dx", dx, tokens, dim, ld_dx, e));
  if (dw_gate) {
    ISOLOCO_TRY(check_matrix("dw_gate", dw_gate, hidden, dim, ld_dw, e));
    ISOLOCO_TRY(check_matrix("dw_up", dw_up, hidden, dim, ld_dw, e));
  }
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const size_t wb = matrix_bytes(hidden, dim, ld_w, e), dwb = matrix_bytes(hidden, dim, ld_dw, e);
  const Range outs[] = {{"dx", dx, matrix_bytes(tokens, dim, ld_dx, e)}, {"dw_gate", dw_gate, dwb},
                        {"dw_up", dw_up, dwb}, {"the workspace", workspace, need}};
  const Range ins[] = {{"x", x, matrix_bytes(tokens, dim, ld_x, e)}, {"w_gate", w_gate, wb}, {"w_up", w_up, wb},
                       {"dout", dout, matrix_bytes(tokens, hidden, ld_dout, e)}};
  ISOLOCO_TRY(check_apart(outs, ins));
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const hipError_t r = BY_TYPES(run_backward, s, x, ld_x, w_gate, w_up, ld_w, dout, ld_dout, dx, ld_dx, dw_gate, dw_up,
                                ld_dw, workspace, st);
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gradient of the gated feed-forward block");
}

}  // extern "C"
