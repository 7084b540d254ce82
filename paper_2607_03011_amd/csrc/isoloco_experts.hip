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
#include "isoloco_vec.h"

namespace isoloco {
namespace {

struct ExpertArgs {
  const void *x, *w, *dout;
  void* out;  // out, dx or dw
  Index offsets, token;
  int64_t tokens, rows, dim, cols;
  int64_t ld_x, ld_w, stride_w, ld_dout, ld_out, stride_out;
  int experts;
};

enum Product { kOut, kDx, kDw };

constexpr int kTile = 64, kDepth = 16;

// Expert e's rows, inside the tensor whatever the offsets; group `experts` is the rows behind the last one's.
__device__ __forceinline__ void rows_of(const ExpertArgs& g, int e, int64_t& begin, int64_t& end) {
  begin = e == 0 ? 0 : min(max(g.offsets.get(e), (int64_t)0), g.rows);
  end = e >= g.experts ? g.rows : max(begin, min(g.offsets.get(e + 1), g.rows));
}

// The group and the first row of the index-th tile of rows; false: there are fewer.
__device__ __forceinline__ bool find_tile(const ExpertArgs& g, int64_t index, int& group, int64_t& first, int64_t& end) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base <= g.experts; base += 64) {
    const int e = base + lane;
    int64_t b = 0, f = 0;
    if (e <= g.experts) rows_of(g, e, b, f);
    const int64_t tiles = (f - b + kTile - 1) / kTile;
    int64_t sum = tiles;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t o = __shfl_up((long long)sum, off, 64);
      if (lane >= off) sum += o;
    }
    const uint64_t past = __ballot(before + sum > index);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      group = base + at;
      first = __shfl((long long)(b + (index - before - (sum - tiles)) * kTile), at, 64);
      end = __shfl((long long)f, at, 64);
      return true;
    }
    before += __shfl((long long)sum, 63, 64);
  }
  return false;
}

template <typename T, Product P>
__global__ void __launch_bounds__(256) expert_kernel(ExpertArgs g, int tiles_n) {
  __shared__ float a[kDepth][kTile + 1], b[kDepth][kTile + 1];
  const int tn = blockIdx.x % tiles_n;
  int64_t tm = blockIdx.x / tiles_n;
  int e;
  int64_t first, end, m0, m_end;
  if (P == kDw) {
    const int tiles_m = (int)((g.cols + kTile - 1) / kTile);
    e = (int)(tm / tiles_m);
    m0 = (tm - (int64_t)e * tiles_m) * kTile;
    m_end = g.cols;
    rows_of(g, e, first, end);
  } else {
    if (!find_tile(g, tm, e, first, end)) return;
    m0 = first;
    m_end = end;
  }
  const int64_t n0 = (int64_t)tn * kTile, n_end = P == kOut ? g.cols : g.dim;
  int64_t depth = P == kOut ? g.dim : P == kDx ? g.cols : end - first;
  if (e >= g.experts) depth = 0;  // rows of no expert: zeros
  const T *x = static_cast<const T*>(g.x), *d = static_cast<const T*>(g.dout);
  const T* w = static_cast<const T*>(g.w) + (e < g.experts ? e : 0) * g.stride_w;
  const auto x_at = [&](int64_t r, int64_t k) -> float {
    const int64_t t = g.token.p ? g.token.get(r) : r;
    return t >= 0 && t < g.tokens ? (float)x[t * g.ld_x + k] : 0.f;
  };
  const auto a_at = [&](int64_t m, int64_t k) -> float {
    if (P == kOut) return x_at(m, k);
    return P == kDx ? (float)d[m * g.ld_dout + k] : (float)d[(first + k) * g.ld_dout + m];
  };
  const auto b_at = [&](int64_t n, int64_t k) -> float {
    if (P == kOut) return (float)w[n * g.ld_w + k];
    return P == kDx ? (float)w[k * g.ld_w + n] : x_at(first + k, n);
  };
  float acc[4][4] = {};
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int64_t k0 = 0; k0 < depth; k0 += kDepth) {
    for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
      const int k = i % kDepth, m = i / kDepth;
      const bool in = k0 + k < depth;
      a[k][m] = in && m0 + m < m_end ? a_at(m0 + m, k0 + k) : 0.f;
      b[k][m] = in && n0 + m < n_end ? b_at(n0 + m, k0 + k) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < kDepth; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[k][ty + 16 * i], b[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
  T* out = static_cast<T*>(g.out) + (P == kDw ? e * g.stride_out : 0);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m < m_end && n < n_end) out[m * g.ld_out + n] = (T)acc[i][j];
    }
}

template <Product P>
hipError_t launch(int32_t dtype, const ExpertArgs& g, hipStream_t st) {
  const int64_t n = P == kOut ? g.cols : g.dim;
  const int tiles_n = (int)((n + kTile - 1) / kTile);
  const int64_t tiles_m = P == kDw ? g.experts * ((g.cols + kTile - 1) / kTile)
                                   : g.rows / kTile + std::min<int64_t>(g.rows, g.experts + 1);
  if (tiles_m == 0) return hipSuccess;
  const dim3 grid((unsigned)(tiles_m * tiles_n));
  if (dtype == ISOLOCO_F32) hipLaunchKernelGGL((expert_kernel<float, P>), grid, dim3(256), 0, st, g, tiles_n);
  else hipLaunchKernelGGL((expert_kernel<__bf16, P>), grid, dim3(256), 0, st, g, tiles_n);
  return hipGetLastError();
}

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

size_t expert_workspace(const ExpertShape&, int32_t) { return 0; }

}  // namespace
}  // namespace isoloco

using namespace isoloco;

extern "C" {

isoloco_status isoloco_expert_matmul_workspace_size(int64_t tokens, int64_t rows, int64_t experts, int64_t dim,
                                                    int64_t cols, int32_t dtype, int32_t flags, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  const ExpertShape s = {tokens, rows, experts, dim, cols, dtype};
  ISOLOCO_TRY(check_shape(s));
  if (flags & ~(ISOLOCO_EXPERTS_BACKWARD | ISOLOCO_EXPERTS_ALIGNED | ISOLOCO_EXPERTS_GATHERED))
    return fail(ISOLOCO_ERR_INVALID_ARG, "flags = %d", flags);
  *bytes = expert_workspace(s, flags);
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
  const size_t need = expert_workspace(s, 0);
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const Operand ins[] = {{"x", x, matrix_bytes(tokens, dim, ld_x, e), e},
                         {"w", w, experts_bytes(s, ld_w, stride_w), e},
                         {"offsets", offsets, (size_t)(experts + 1) * ib, ib},
                         {"token", token, token ? (size_t)rows * ib : 0, ib}};
  const Operand outs[] = {{"out", out, matrix_bytes(rows, cols, ld_out, e), e}, {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_operands(outs, 2, ins, 4));
  ExpertArgs g = {};
  g.x = x;
  g.w = w;
  g.out = out;
  g.offsets = {offsets, index_type == ISOLOCO_I64};
  g.token = {token, index_type == ISOLOCO_I64};
  g.tokens = tokens;
  g.rows = rows;
  g.dim = dim;
  g.cols = cols;
  g.ld_x = ld_x;
  g.ld_w = ld_w;
  g.stride_w = stride_w;
  g.ld_out = ld_out;
  g.experts = (int)experts;
  const hipError_t r = launch<kOut>(dtype, g, static_cast<hipStream_t>(hip_stream));
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
  const size_t need = expert_workspace(s, ISOLOCO_EXPERTS_BACKWARD);
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
  ExpertArgs g = {};
  g.x = x;
  g.w = w;
  g.dout = dout;
  g.offsets = {offsets, index_type == ISOLOCO_I64};
  g.token = {token, index_type == ISOLOCO_I64};
  g.tokens = tokens;
  g.rows = rows;
  g.dim = dim;
  g.cols = cols;
  g.ld_x = ld_x;
  g.ld_w = ld_w;
  g.stride_w = stride_w;
  g.ld_dout = ld_dout;
  g.experts = (int)experts;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t r = hipSuccess;
  if (dx && rows) {
    g.out = dx;
    g.ld_out = ld_dx;
    r = launch<kDx>(dtype, g, st);
  }
  if (r == hipSuccess && dw) {
    g.out = dw;
    g.ld_out = ld_dw;
    g.stride_out = stride_dw;
    r = launch<kDw>(dtype, g, st);
  }
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gradient of products grouped by expert");
}

}  // extern "C"
