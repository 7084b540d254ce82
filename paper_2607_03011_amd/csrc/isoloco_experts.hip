// Products grouped by expert.  Expert e has rows offsets[e] .. offsets[e + 1] - 1 of the
// grouped order; row r's input is x[token[r]] (or x[r] without token):
//
//   out[r] = x_r w[e]^T,   dx[r] = dout[r] w[e],   dw[e] = sum over its rows of dout[r]^T x_r
//
// Rows of no expert give zeros.  The sizes are read on the device: a launch has as many
// workgroups as the worst case needs, and each finds its tile among the experts' rows.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_experts.h"
#include "isoloco_ffn.h"
#include "isoloco_lds.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

struct ExpertShape {
  int64_t tokens, rows, experts, dim, cols;
  int32_t dtype;
};

isoloco_status check_shape(const ExpertShape& s) {
  // a tile's rows are addressed with offsets of 32 bits: 256 rows of 2 bytes times this
  constexpr int64_t most = ((int64_t)1 << 22) - 64;
  if (s.rows < 0 || s.rows > kMaxExtent - 1 || s.tokens < 0 || s.tokens > kMaxExtent - 1 || s.dim < 1 || s.dim > most ||
      s.cols < 1 || s.cols > most)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of %lld tokens, dim %lld, cols %lld", (long long)s.rows,
                (long long)s.tokens, (long long)s.dim, (long long)s.cols);
  if (s.experts < 1 || s.experts > ISOLOCO_MAX_EXPERTS)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld experts, of 1 to %d", (long long)s.experts, ISOLOCO_MAX_EXPERTS);
  if (!is_dtype(s.dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", s.dtype);
  return ISOLOCO_OK;
}

// An operand of `experts` matrices, stride elements apart.
isoloco_status check_experts(const char* name, const void* p, const ExpertShape& s, int64_t ld, int64_t stride) {
  ISOLOCO_TRY(check_matrix(name, p, s.cols, s.dim, ld, dtype_bytes(s.dtype)));
  if (s.experts > 1 && (stride < (s.cols - 1) * ld + s.dim || stride > (int64_t)1 << 44))
    return fail(ISOLOCO_ERR_INVALID_ARG, "%s: matrices %lld elements apart, of %lld rows", name, (long long)stride,
                (long long)s.cols);
  return ISOLOCO_OK;
}
size_t experts_bytes(const ExpertShape& s, int64_t ld, int64_t stride) {
  return (size_t)(s.experts - 1) * stride * dtype_bytes(s.dtype) + matrix_bytes(s.cols, s.dim, ld, dtype_bytes(s.dtype));
}

// What a call hands to the tile products, and where its copies lie in the workspace.
struct CallPlan {
  bool copy_x, copy_w, copy_d;  // operands that the tiles do not read where they are
  bool gather_x;                // the copy of x has the grouped rows
  size_t x, w, d, partial, bytes;
};

bool tile_rows(const void* p, int64_t cols, int64_t ld) {
  return aligned_to(p, 16) && ((cols | ld) & 7) == 0 && ld <= (1 << 22);
}

// x_ok, w_ok, d_ok: the operand may be read where it is.  x is read by the forward product and
// by dw, w by the forward product and by dx.
CallPlan call_plan(const ExpertShape& s, bool gathered, bool dx, bool dw, bool x_ok, bool w_ok, bool d_ok, int64_t ld_x) {
  CallPlan p = {};
  const bool f32 = s.dtype == ISOLOCO_F32, back = dx || dw;
  const size_t parts = f32 ? kFfnParts : 1;
  const int64_t dim = ffn_pad(s.dim), cols = ffn_pad(s.cols);
  const auto take = [&](size_t bytes) {
    const size_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  p.copy_x = (dw || !back) && (f32 || !x_ok);
  p.copy_w = (dx || !back) && (f32 || !w_ok);
  p.copy_d = back && (f32 || !d_ok);
  // gathered rows are addressed in 32 bits
  if (gathered && (dw || !back) && 2 * s.tokens * (p.copy_x ? dim : ld_x) > (int64_t)kMostBytes) p.copy_x = p.gather_x = true;
  if (p.copy_x) p.x = take(2 * parts * (p.gather_x || !gathered ? s.rows : s.tokens) * dim);
  if (p.copy_w) p.w = take(2 * parts * s.experts * s.cols * dim);
  if (p.copy_d) p.d = take(2 * parts * s.rows * cols);
  size_t partial = 0;
  if (!back) partial = expert_partial_bytes(kOut, f32, s.rows, s.experts, 0, s.cols, s.dim);
  if (dx) partial = std::max(partial, expert_partial_bytes(kDx, f32, s.rows, s.experts, 0, s.dim, s.cols));
  if (dw) partial = std::max(partial, expert_partial_bytes(kDw, f32, s.rows, s.experts, s.cols, s.dim, 0));
  p.partial = take(partial);
  return p;
}

struct CopyJob {
  const void* src;
  uint16_t* dst;
  Index token;     // p NULL: rows as they lie
  int64_t tokens;  // of src, where token is given: others are rows of zeros
  int64_t rows, per_matrix, cols, ld, stride, ld_dst;
};
struct CopyArgs {
  CopyJob job[3];
};

// Matrices as bfloat16 with rows of ld_dst = ffn_pad(cols), zeros past cols; float32 as three
// parts, one after the other.  One thread per 8 elements of a row.
template <typename T>
__global__ void __launch_bounds__(256) expert_copy_kernel(CopyArgs c) {
  const CopyJob& j = c.job[blockIdx.y];
  const int64_t per_row = j.ld_dst / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < j.rows * per_row; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row, col = (i - row * per_row) * 8;
    int64_t from = row;
    bool in = true;
    if (j.token.p) {
      from = j.token.get(row);
      in = from >= 0 && from < j.tokens;
    }
    const int64_t matrix = from / j.per_matrix;
    const T* p = static_cast<const T*>(j.src) + matrix * j.stride + (from - matrix * j.per_matrix) * j.ld + col;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e += Vec<T>::N) load_piece<T>(p + e, in ? j.cols - col - e : 0, x + e);
    uint16_t* q = j.dst + row * j.ld_dst + col;
#pragma unroll
    for (int part = 0; part < (sizeof(T) == 4 ? kFfnParts : 1); ++part) {
      const u32x4 v = pack<__bf16>(x);
      float r[8];
      unpack<__bf16>(v, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] -= r[e];
      *reinterpret_cast<u32x4*>(q + part * j.rows * j.ld_dst) = v;
    }
  }
}

// The operands of the tile products, copied where they have to be.
struct Operands {
  const uint16_t *x, *w, *d;
  int64_t ld_x, ld_w, ld_d, stride_w, part_x, part_w, part_d;
  Index token;
  int64_t tokens;
};

struct Call {
  ExpertShape s;
  const void *x, *w, *d;
  int64_t ld_x, ld_w, stride_w, ld_d;
  Index offsets, token;
};

Operands copy_operands(const Call& c, const CallPlan& p, char* ws, hipStream_t st) {
  const ExpertShape& s = c.s;
  const int64_t dim = ffn_pad(s.dim), cols = ffn_pad(s.cols);
  Operands o = {};
  o.x = static_cast<const uint16_t*>(c.x);
  o.w = static_cast<const uint16_t*>(c.w);
  o.d = static_cast<const uint16_t*>(c.d);
  o.ld_x = c.ld_x;
  o.ld_w = c.ld_w;
  o.ld_d = c.ld_d;
  o.stride_w = c.stride_w;
  o.token = c.token;
  o.tokens = s.tokens;
  CopyArgs a = {};
  int n = 0;
  int64_t most = 0;
  const auto add = [&](const void* src, size_t at, int64_t rows, int64_t per_matrix, int64_t width, int64_t ld,
                       int64_t stride, int64_t ld_dst, Index token) {
    a.job[n++] = {src, reinterpret_cast<uint16_t*>(ws + at), token, s.tokens, rows, per_matrix, width, ld, stride, ld_dst};
    most = std::max(most, rows * (ld_dst / 8));
    return reinterpret_cast<const uint16_t*>(ws + at);
  };
  const int64_t x_rows = p.gather_x || !c.token.p ? s.rows : s.tokens, whole = kMaxExtent;
  if (p.copy_x) {
    o.x = add(c.x, p.x, x_rows, whole, s.dim, c.ld_x, 0, dim, p.gather_x ? c.token : Index{});
    o.ld_x = dim;
    o.part_x = x_rows * dim;
    if (p.gather_x) o.token = {};
  }
  if (p.copy_w) {
    o.w = add(c.w, p.w, s.experts * s.cols, s.cols, s.dim, c.ld_w, c.stride_w, dim, Index{});
    o.ld_w = dim;
    o.stride_w = s.cols * dim;
    o.part_w = s.experts * s.cols * dim;
  }
  if (p.copy_d) {
    o.d = add(c.d, p.d, s.rows, whole, s.cols, c.ld_d, 0, cols, Index{});
    o.ld_d = cols;
    o.part_d = s.rows * cols;
  }
  const unsigned grid = (unsigned)std::min<int64_t>((most + 255) / 256, 1 << 14);
  if (grid) {
    if (s.dtype == ISOLOCO_F32) hipLaunchKernelGGL(expert_copy_kernel<float>, dim3(grid, n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(expert_copy_kernel<__bf16>, dim3(grid, n), dim3(256), 0, st, a);
  }
  return o;
}

ExpertArgs args_of(const Call& c, const Operands& o, const CallPlan& p, char* ws) {
  ExpertArgs g = {};
  g.groups = {c.offsets, c.s.rows, (int)c.s.experts};
  g.token = o.token;
  g.tokens = o.tokens;
  g.partial = reinterpret_cast<float*>(ws + p.partial);
  return g;
}

hipError_t run_forward(const Call& c, const CallPlan& p, void* out, int64_t ld_out, char* ws, hipStream_t st) {
  const Operands o = copy_operands(c, p, ws, st);
  ExpertArgs g = args_of(c, o, p, ws);
  g.a = o.x;
  g.ld_a = o.ld_x;
  g.part_a = o.part_x;
  g.b = o.w;
  g.ld_b = o.ld_w;
  g.part_b = o.part_w;
  g.stride_b = o.stride_w;
  g.n = c.s.cols;
  g.k = p.copy_x && p.copy_w ? ffn_pad(c.s.dim) : (c.s.dim + 7) / 8 * 8;
  g.out = out;
  g.ld_out = ld_out;
  return launch_expert_tiles(kOut, c.s.dtype == ISOLOCO_F32, g, st);
}

hipError_t run_backward(const Call& c, const CallPlan& p, void* dx, int64_t ld_dx, void* dw, int64_t ld_dw,
                        int64_t stride_dw, char* ws, hipStream_t st) {
  const bool f32 = c.s.dtype == ISOLOCO_F32;
  const int64_t dim = ffn_pad(c.s.dim), cols = ffn_pad(c.s.cols);
  const Operands o = copy_operands(c, p, ws, st);
  ExpertArgs g = args_of(c, o, p, ws);
  g.a = o.d;
  g.ld_a = o.ld_d;
  g.part_a = o.part_d;
  g.n = c.s.dim;
  hipError_t r = hipSuccess;
  if (dx) {
    ExpertArgs h = g;
    h.token = {};
    h.b = o.w;
    h.ld_b = o.ld_w;
    h.part_b = o.part_w;
    h.stride_b = o.stride_w;
    h.cols_b = p.copy_w ? dim : c.s.dim;
    h.k = c.s.cols;
    h.out = dx;
    h.ld_out = ld_dx;
    r = launch_expert_tiles(kDx, f32, h, st);
  }
  if (r == hipSuccess && dw) {
    g.b = o.x;
    g.ld_b = o.ld_x;
    g.part_b = o.part_x;
    g.cols_a = p.copy_d ? cols : c.s.cols;
    g.cols_b = p.copy_x ? dim : c.s.dim;
    g.m = c.s.cols;
    g.out = dw;
    g.ld_out = ld_dw;
    g.stride_out = stride_dw;
    r = launch_expert_tiles(kDw, f32, g, st);
  }
  return r;
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

extern "C" {

isoloco_status isoloco_expert_matmul_workspace_size(int64_t tokens, int64_t rows, int64_t experts, int64_t dim,
                                                    int64_t cols, int64_t ld_x, int32_t dtype, int32_t flags,
                                                    size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  const ExpertShape s = {tokens, rows, experts, dim, cols, dtype};
  ISOLOCO_TRY(check_shape(s));
  if (flags & ~(ISOLOCO_EXPERTS_BACKWARD | ISOLOCO_EXPERTS_ALIGNED | ISOLOCO_EXPERTS_GATHERED))
    return fail(ISOLOCO_ERR_INVALID_ARG, "flags = %d", flags);
  const bool ok = flags & ISOLOCO_EXPERTS_ALIGNED, back = flags & ISOLOCO_EXPERTS_BACKWARD;
  *bytes = call_plan(s, flags & ISOLOCO_EXPERTS_GATHERED, back, back, ok, ok, ok, ld_x).bytes;
  return ISOLOCO_OK;
}

isoloco_status isoloco_expert_matmul(const void* x, int64_t ld_x, int64_t tokens, const void* token, const void* w,
                                     int64_t ld_w, int64_t stride_w, int32_t dtype, const void* offsets,
                                     int32_t index_type, int64_t experts, int64_t rows, int64_t dim, int64_t cols,
                                     void* out, int64_t ld_out, void* workspace, size_t workspace_bytes,
                                     void* hip_stream) {
  const ExpertShape s = {tokens, rows, experts, dim, cols, dtype};
  ISOLOCO_TRY(check_shape(s));
  if (!is_index_type(index_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type %d", index_type);
  if (!token && tokens != rows) return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of x, %lld wanted", (long long)tokens, (long long)rows);
  if (rows == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type);
  ISOLOCO_TRY(check_matrix("x", x, tokens, dim, ld_x, e));
  ISOLOCO_TRY(check_experts("w", w, s, ld_w, stride_w));
  ISOLOCO_TRY(check_matrix("out", out, rows, cols, ld_out, e));
  const CallPlan p = call_plan(s, token, false, false, tile_rows(x, dim, ld_x),
                         tile_rows(w, dim, ld_w) && (experts == 1 || (stride_w & 7) == 0), true, ld_x);
  const size_t need = p.bytes;
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const Operand ins[] = {{"x", x, matrix_bytes(tokens, dim, ld_x, e), e},
                         {"w", w, experts_bytes(s, ld_w, stride_w), e},
                         {"offsets", offsets, (size_t)(experts + 1) * ib, ib},
                         {"token", token, token ? (size_t)rows * ib : 0, ib}};
  const Operand outs[] = {{"out", out, matrix_bytes(rows, cols, ld_out, e), e}, {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_operands(outs, 2, ins, 4));
  const bool wide = index_type == ISOLOCO_I64;
  const Call c = {s, x, w, nullptr, ld_x, ld_w, stride_w, 0, {offsets, wide}, {token, wide}};
  const hipError_t r = run_forward(c, p, out, ld_out, static_cast<char*>(workspace), static_cast<hipStream_t>(hip_stream));
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "products grouped by expert");
}

isoloco_status isoloco_expert_matmul_backward(const void* x, int64_t ld_x, int64_t tokens, const void* token,
                                              const void* w, int64_t ld_w, int64_t stride_w, int32_t dtype,
                                              const void* offsets, int32_t index_type, int64_t experts, int64_t rows,
                                              int64_t dim, int64_t cols, const void* dout, int64_t ld_dout, void* dx,
                                              int64_t ld_dx, void* dw, int64_t ld_dw, int64_t stride_dw,
                                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  const ExpertShape s = {tokens, rows, experts, dim, cols, dtype};
  ISOLOCO_TRY(check_shape(s));
  if (!is_index_type(index_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type %d", index_type);
  if (!token && tokens != rows) return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of x, %lld wanted", (long long)tokens, (long long)rows);
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type);
  if (dw) {
    ISOLOCO_TRY(check_matrix("x", x, tokens, dim, ld_x, e));
    ISOLOCO_TRY(check_experts("dw", dw, s, ld_dw, stride_dw));
  }
  if (dx && rows) {
    ISOLOCO_TRY(check_experts("w", w, s, ld_w, stride_w));
    ISOLOCO_TRY(check_matrix("dx", dx, rows, dim, ld_dx, e));
  }
  ISOLOCO_TRY(check_matrix("dout", dout, rows, cols, ld_dout, e));
  if (rows == 0) dx = nullptr;
  const CallPlan p = call_plan(s, token, dx, dw, tile_rows(x, dim, ld_x),
                         tile_rows(w, dim, ld_w) && (experts == 1 || (stride_w & 7) == 0), tile_rows(dout, cols, ld_dout), ld_x);
  const size_t need = p.bytes;
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const Operand ins[] = {{"x", x, dw ? matrix_bytes(tokens, dim, ld_x, e) : 0, e},
                         {"w", w, dx && rows ? experts_bytes(s, ld_w, stride_w) : 0, e},
                         {"dout", dout, matrix_bytes(rows, cols, ld_dout, e), e},
                         {"offsets", offsets, (size_t)(experts + 1) * ib, ib},
                         {"token", token, token && dw ? (size_t)rows * ib : 0, ib}};
  const Operand outs[] = {{"dx", dx, dx ? matrix_bytes(rows, dim, ld_dx, e) : 0, e},
                          {"dw", dw, dw ? experts_bytes(s, ld_dw, stride_dw) : 0, e},
                          {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_operands(outs, 3, ins, 5));
  const bool wide = index_type == ISOLOCO_I64;
  const Call c = {s, x, w, dout, ld_x, ld_w, stride_w, ld_dout, {offsets, wide}, {token, wide}};
  const hipError_t r = run_backward(c, p, dx, ld_dx, dw, ld_dw, stride_dw, static_cast<char*>(workspace),
                                    static_cast<hipStream_t>(hip_stream));
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gradient of products grouped by expert");
}

}  // extern "C"
