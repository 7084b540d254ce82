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
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef floatx4 floatx4_any __attribute__((aligned(4)));

// ---------------------------------------------------------------------------
// Few tokens
// ---------------------------------------------------------------------------
//
// A product of few rows is bounded by the weights' bytes: every weight is loaded once,
// from memory into the registers that the MFMA reads (16 weight rows against 16
// tokens), and the workgroup's waves split dim so that enough loads are in flight.

// The values of k that a lane holds of one row, 16 bytes: its MFMA operands.
template <typename T>
struct Lane {
  static constexpr int N = 16 / sizeof(T);
  alignas(16) T v[N];
  __device__ __forceinline__ void load(const T* p, int64_t left) {
    if (left >= N) {
      *reinterpret_cast<u32x4*>(v) = *reinterpret_cast<const u32x4_any*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < left ? p[e] : (T)0.f;
    }
  }
};
__device__ __forceinline__ floatx4 multiply(const Lane<__bf16>& a, const Lane<__bf16>& b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8_t*>(a.v),
                                                 *reinterpret_cast<const bf16x8_t*>(b.v), c, 0, 0, 0);
}
// (which k a lane's e-th value stands for is the same in both operands)
__device__ __forceinline__ floatx4 multiply(const Lane<float>& a, const Lane<float>& b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// Up to few_most() tokens come here, the others go to the tiles.  Both sides measured, us a
// call of a graph, weights in a cache, here / tiles:
//                           16 tokens    17           32           33           64
//   bfloat16   768 x 2048   3.9 / 8.3    4.3 / 8.2    4.6 / 8.8    5.4 / 8.7    6.1 / 9.8
//             1000 x 2777   4.9 / 9.3    6.1 / 9.3    6.4 / 10.1   8.4 / 10.3   9.6 / 12.1
//             2048 x 5632   13.5 / 15.1  14.7 / 15.1  18.7 / 15.9  21.4 / 16.3  29.7 / 18.0
//   float32    768 x 2048   5.3 / 28.7   5.9 / 29.0   6.6 / 28.0   8.5 / 28.3   9.9 / 27.9
//             2048 x 5632   24.5 / 81.7  26.8 / 82.1  34.7 / 83.2  47.4 / 83.6  57.8 / 88.8
// One line for every width: the wide bfloat16 block is better off with the tiles from 18
// tokens on, the narrow ones here up to 64.
constexpr int kFewWaves = 8;
constexpr int64_t few_most(int32_t dtype) { return dtype == ISOLOCO_BF16 ? 32 : 64; }

// 8 hidden rows per workgroup, up to 16 NT tokens.  The gate's rows are the first 8 of an
// MFMA operand, the up projection's the others.  (16 rows of each per workgroup: 352
// workgroups for 5632, two on some CUs and one on others, 14.3 us for one token of 2048
// against 11.6.)
template <typename T, int ACT, int NT>
__global__ void __launch_bounds__(64 * kFewWaves) ffn_few_kernel(const T* x, int64_t ld_x, const T* wg, const T* wu,
                                                                int64_t ld_w, int tokens, int64_t dim, int64_t hidden,
                                                                T* out, int64_t ld_out) {
  constexpr int N = Lane<T>::N, kStep = 4 * N;  // k values of one step
  __shared__ floatx4 sums[kFewWaves][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, kl = (lane >> 4) * N;
  const int64_t h0 = (int64_t)blockIdx.x * 8;
  // rows past the matrices are their last ones again: their outputs are not stored
  const T* pw = (row < 8 ? wg : wu) + min(h0 + (row & 7), hidden - 1) * ld_w + kl;
  const T* px[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) px[n] = x + (int64_t)min(16 * n + row, tokens - 1) * ld_x + kl;
  floatx4 s[NT] = {};
  // kAhead steps' loads are in flight at a time
  constexpr int kAhead = 4;
  constexpr int64_t kStride = kFewWaves * kStep;
  int64_t k = (int64_t)wave * kStep;
  for (; k + (kAhead - 1) * kStride + kStep <= dim; k += kAhead * kStride) {
    Lane<T> a[kAhead], c[kAhead][NT];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      a[i].load(pw + k + i * kStride, N);
#pragma unroll
      for (int n = 0; n < NT; ++n) c[i][n].load(px[n] + k + i * kStride, N);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n] = multiply(a[i], c[i][n], s[n]);
  }
  for (; k < dim; k += kStride) {
    const int64_t left = dim - k - kl;
    Lane<T> a, c;
    a.load(pw + k, left);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      c.load(px[n] + k, left);
      s[n] = multiply(a, c, s[n]);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) sums[wave][n][lane] = s[n];
  __syncthreads();
  // lanes l < 32 hold rows 4 (l / 16) .. + 3 of the gate for token l % 16, lanes l + 32 the
  // same of the up projection; wave n finishes 16 tokens
  if (wave >= NT || lane >= 32) return;
  floatx4 gate = {}, up = {};
  for (int w = 0; w < kFewWaves; ++w) {
    gate += sums[w][wave][lane];
    up += sums[w][wave][lane + 32];
  }
  const int t = 16 * wave + (lane & 15);
  if (t >= tokens) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t j = h0 + 4 * (lane >> 4) + e;
    float f, df;
    activate<ACT, sizeof(T) == 4>(gate[e], f, df);
    if (j < hidden) out[(int64_t)t * ld_out + j] = (T)(f * up[e]);
  }
}

// ---------------------------------------------------------------------------
// Copies for the tile products
// ---------------------------------------------------------------------------

struct CopyArgs {
  const void* src[3];
  uint16_t* dst[3];
  int64_t rows[3], ld_src[3];
  int64_t cols, ld_dst;
  int n;
};

// Matrices as bfloat16 with rows of ld_dst = ffn_pad(cols), zeros past cols; float32 as
// three parts, one after the other.  One thread per 8 elements of a row.
template <typename T>
__global__ void __launch_bounds__(256) ffn_copy_kernel(CopyArgs c) {
  const int m = blockIdx.y;
  const int64_t per_row = c.ld_dst / 8, rows = c.rows[m];
  const T* src = static_cast<const T*>(c.src[m]);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per_row; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row, col = (i - row * per_row) * 8;
    const T* p = src + row * c.ld_src[m] + col;
    const int64_t left = c.cols - col;
    uint16_t* q = c.dst[m] + row * c.ld_dst + col;
    if constexpr (sizeof(T) == 2) {
      Lane<__bf16> v;
      v.load(p, left);
      *reinterpret_cast<u32x4*>(q) = *reinterpret_cast<const u32x4*>(v.v);
    } else {
      Lane<float> v[2];
      v[0].load(p, left);
      v[1].load(p + 4, left - 4);
#pragma unroll
      for (int part = 0; part < kFfnParts; ++part) {
        bf16x8_t b;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          b[e] = (__bf16)v[e / 4].v[e % 4];
          v[e / 4].v[e % 4] -= (float)b[e];
        }
        *reinterpret_cast<bf16x8_t*>(q + part * rows * c.ld_dst) = b;
      }
    }
  }
}

struct FfnShape {
  int64_t tokens, dim, hidden;
  int32_t dtype, act;
};

// What a call hands to the tile products, and where its copies lie in the workspace.
struct FfnPlan {
  bool few;                        // ffn_few_kernel
  bool copy_x, copy_w;             // operands that the tiles do not read where they are
  size_t x, wg, wu, da, du, partial, bytes;  // offsets in the workspace
};

// the tile products load whole 16-byte pieces of rows
bool tile_rows(const void* p, int64_t ld) { return aligned_to(p, 16) && (ld & 7) == 0 && ld <= (1 << 22); }

// `x_ok`, `w_ok`: the operand may be read where it is.
FfnPlan plan_of(const FfnShape& s, bool backward, bool x_ok, bool w_ok) {
  FfnPlan p = {};
  const bool f32 = s.dtype == ISOLOCO_F32;
  p.few = !backward && s.tokens <= few_most(s.dtype);
  if (p.few) return p;
  p.copy_x = f32 || !x_ok || (s.dim & 7);
  p.copy_w = f32 || !w_ok || (s.dim & 7);
  const size_t parts = f32 ? kFfnParts : 1, row = 2 * (size_t)ffn_pad(s.dim) * parts;
  const auto take = [&](size_t bytes) {
    const size_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  if (p.copy_x) p.x = take(row * s.tokens);
  if (p.copy_w) {
    p.wg = take(row * s.hidden);
    p.wu = take(row * s.hidden);
  }
  size_t partial = ffn_projections_partial_bytes(backward ? kInner : kForward, f32, s.tokens, s.hidden, s.dim);
  if (backward) {
    const size_t inner = 2 * (size_t)ffn_pad(s.tokens) * (size_t)ffn_pad(s.hidden) * parts;
    p.da = take(inner);
    p.du = take(inner);
    partial = std::max(partial, ffn_gradients_partial_bytes(f32, s.tokens, s.dim, s.hidden));
  }
  p.partial = take(partial);
  return p;
}

template <typename T, int ACT, int NT>
void launch_few(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, void* out,
                int64_t ld_out, hipStream_t st) {
  hipLaunchKernelGGL((ffn_few_kernel<T, ACT, NT>), dim3((unsigned)((s.hidden + 7) / 8)), dim3(64 * kFewWaves), 0, st,
                     static_cast<const T*>(x), ld_x, static_cast<const T*>(wg), static_cast<const T*>(wu), ld_w,
                     (int)s.tokens, s.dim, s.hidden, static_cast<T*>(out), ld_out);
}

// The operands of the tile products, copied where they have to be.
struct TileOperands {
  const uint16_t *x, *wg, *wu;
  int64_t ld_x, ld_w, part_x, part_w;
  int64_t k;  // dim, padded if both are copies
};
template <typename T>
TileOperands copy_operands(const FfnShape& s, const FfnPlan& p, const void* x, int64_t ld_x, const void* wg,
                           const void* wu, int64_t ld_w, char* ws, hipStream_t st) {
  const int64_t ld = ffn_pad(s.dim);
  TileOperands o = {static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(wg), static_cast<const uint16_t*>(wu),
                    ld_x, ld_w, s.tokens * ld, s.hidden * ld, p.copy_x && p.copy_w ? ld : s.dim};
  CopyArgs c = {};
  c.cols = s.dim;
  c.ld_dst = ld;
  const auto add = [&](const uint16_t*& from, int64_t& ld_from, int64_t rows, size_t at) {
    c.src[c.n] = from;
    c.ld_src[c.n] = ld_from;
    c.rows[c.n] = rows;
    c.dst[c.n++] = reinterpret_cast<uint16_t*>(ws + at);
    from = reinterpret_cast<const uint16_t*>(ws + at);
  };
  if (p.copy_x) add(o.x, o.ld_x, s.tokens, p.x);
  if (p.copy_w) {
    add(o.wg, o.ld_w, s.hidden, p.wg);
    add(o.wu, o.ld_w, s.hidden, p.wu);
  }
  if (p.copy_x) o.ld_x = ld;
  if (p.copy_w) o.ld_w = ld;
  if (c.n) {
    const int64_t items = std::max(p.copy_x ? s.tokens : 0, p.copy_w ? s.hidden : 0) * (ld / 8);
    const unsigned grid = (unsigned)std::min<int64_t>((items + 255) / 256, 1 << 20);
    if (grid) hipLaunchKernelGGL(ffn_copy_kernel<T>, dim3(grid, c.n), dim3(256), 0, st, c);
  }
  return o;
}

template <typename T, int ACT>
hipError_t run_forward(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w,
                       void* out, int64_t ld_out, void* ws, hipStream_t st) {
  const FfnPlan p = plan_of(s, false, tile_rows(x, ld_x), tile_rows(wg, ld_w) && tile_rows(wu, ld_w));
  if (p.few) {
    if (s.tokens <= 16) launch_few<T, ACT, 1>(s, x, ld_x, wg, wu, ld_w, out, ld_out, st);
    else if (s.tokens <= 32) launch_few<T, ACT, 2>(s, x, ld_x, wg, wu, ld_w, out, ld_out, st);
    else if constexpr (sizeof(T) == 4) launch_few<T, ACT, 4>(s, x, ld_x, wg, wu, ld_w, out, ld_out, st);
    return hipGetLastError();
  }
  const TileOperands o = copy_operands<T>(s, p, x, ld_x, wg, wu, ld_w, static_cast<char*>(ws), st);
  FfnArgs g = {};
  g.a[0] = o.x;
  g.b[0] = o.wg;
  g.b[1] = o.wu;
  g.ld_a = o.ld_x;
  g.ld_b = o.ld_w;
  g.part_a = o.part_x;
  g.part_b = o.part_w;
  g.m = s.tokens;
  g.n = s.hidden;
  g.k = o.k;
  g.out[0] = out;
  g.ld_out = ld_out;
  g.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + p.partial);
  return launch_ffn_projections(kForward, ACT, sizeof(T) == 4, g, st);
}

template <typename T, int ACT>
hipError_t run_backward(const FfnShape& s, const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w,
                        const void* dout, int64_t ld_dout, void* dx, int64_t ld_dx, void* dwg, void* dwu,
                        int64_t ld_dw, void* ws, hipStream_t st) {
  constexpr bool f32 = sizeof(T) == 4;
  char* base = static_cast<char*>(ws);
  const FfnPlan p = plan_of(s, true, tile_rows(x, ld_x), tile_rows(wg, ld_w) && tile_rows(wu, ld_w));
  const TileOperands o = copy_operands<T>(s, p, x, ld_x, wg, wu, ld_w, base, st);
  const int64_t ld = ffn_pad(s.hidden), part = ffn_pad(s.tokens) * ld, cols = ffn_pad(s.dim);
  uint16_t* da = reinterpret_cast<uint16_t*>(base + p.da);
  uint16_t* du = reinterpret_cast<uint16_t*>(base + p.du);
  FfnArgs g = {};
  g.a[0] = o.x;
  g.b[0] = o.wg;
  g.b[1] = o.wu;
  g.ld_a = o.ld_x;
  g.ld_b = o.ld_w;
  g.part_a = o.part_x;
  g.part_b = o.part_w;
  g.m = s.tokens;
  g.n = s.hidden;
  g.k = o.k;
  g.out[0] = da;
  g.out[1] = du;
  g.ld_out = ld;
  g.part_out = part;
  g.dh = dout;
  g.ld_dh = ld_dout;
  g.partial = reinterpret_cast<float*>(base + p.partial);
  const hipError_t e = launch_ffn_projections(kInner, ACT, f32, g, st);
  if (e != hipSuccess) return e;
  g = {};
  g.a[0] = da;
  g.a[1] = du;
  g.ld_a = ld;
  g.part_a = part;
  g.n = s.dim;
  g.partial = reinterpret_cast<float*>(base + p.partial);
  FfnArgs sum = g, pair = g;
  sum.b[0] = o.wg;
  sum.b[1] = o.wu;
  sum.ld_b = o.ld_w;
  sum.part_b = o.part_w;
  sum.cols_b = p.copy_w ? cols : s.dim;
  sum.m = s.tokens;
  sum.k = s.hidden;
  sum.out[0] = dx;
  sum.ld_out = ld_dx;
  pair.b[0] = pair.b[1] = o.x;
  pair.ld_b = o.ld_x;
  pair.part_b = o.part_x;
  pair.cols_b = p.copy_x ? cols : s.dim;
  pair.m = s.hidden;
  pair.k = s.tokens;
  pair.out[0] = dwg;
  pair.out[1] = dwu;
  pair.ld_out = ld_dw;
  return launch_ffn_gradients(f32, dx ? &sum : nullptr, dwg ? &pair : nullptr, st);
}

isoloco_status check_shape(const FfnShape& s) {
  // a tile's rows are addressed with offsets of 32 bits: 256 rows of 2 bytes times this
  constexpr int64_t most = ((int64_t)1 << 22) - kFfnPad;
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
                                                int32_t flags, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  const FfnShape s = {tokens, dim, hidden, dtype, ISOLOCO_ACT_SILU};
  ISOLOCO_TRY(check_shape(s));
  if (flags & ~(ISOLOCO_FFN_BACKWARD | ISOLOCO_FFN_ALIGNED)) return fail(ISOLOCO_ERR_INVALID_ARG, "flags = %d", flags);
  const bool ok = flags & ISOLOCO_FFN_ALIGNED;
  *bytes = plan_of(s, flags & ISOLOCO_FFN_BACKWARD, ok, ok).bytes;
  return ISOLOCO_OK;
}

isoloco_status isoloco_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w,
                                 int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden, int32_t act, void* out,
                                 int64_t ld_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const FfnShape s = {tokens, dim, hidden, dtype, act};
  ISOLOCO_TRY(check_shape(s));
  if (tokens == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), need = plan_of(s, false, tile_rows(x, ld_x), tile_rows(w_gate, ld_w) && tile_rows(w_up, ld_w)).bytes;
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
  const hipError_t r = BY_TYPES(run_forward, s, x, ld_x, w_gate, w_up, ld_w, out, ld_out, workspace, st);
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gated feed-forward block");
}

isoloco_status isoloco_gated_ffn_backward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up,
                                          int64_t ld_w, int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden,
                                          int32_t act, const void* dout, int64_t ld_dout, void* dx, int64_t ld_dx,
                                          void* dw_gate, void* dw_up, int64_t ld_dw, void* workspace,
                                          size_t workspace_bytes, void* hip_stream) {
  const FfnShape s = {tokens, dim, hidden, dtype, act};
  ISOLOCO_TRY(check_shape(s));
  const size_t e = dtype_bytes(dtype), need = plan_of(s, true, tile_rows(x, ld_x), tile_rows(w_gate, ld_w) && tile_rows(w_up, ld_w)).bytes;
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
