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
  // 64 experts' tiles are counted in 32 bits (splits are of few tiles)
  const int64_t dims = (s.dim + 127) / 128, cols = (s.cols + 127) / 128;
  if ((s.rows / 128 + std::min(s.rows, s.experts)) * std::max(dims, cols) > 1 << 24 ||
      dims * cols > 1 << 24)
    return fail(ISOLOCO_ERR_UNSUPPORTED, "too many tiles: %lld rows, %lld experts of %lld x %lld", (long long)s.rows,
                (long long)s.experts, (long long)s.cols, (long long)s.dim);
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

// ---------------------------------------------------------------------------
// Few rows an expert
// ---------------------------------------------------------------------------
//
// Products of few rows are bounded by the weights' bytes: a workgroup takes 16 rows of an
// expert's weights, which go from memory into the registers that the MFMA reads, and its
// waves split dim so that enough loads are in flight.  Experts without rows are not read.
// Any alignment, float32 as it is: no copies.

struct FewArgs {
  Groups groups;
  Index token;
  int64_t tokens, dim, cols, ld_x, ld_w, stride_w, ld_out;
};

constexpr int kFewWaves = 8;

// The values of k that a lane holds of one row, 16 bytes: its MFMA operands.  (Which k a lane's
// e-th value stands for is the same in both operands.)
__device__ __forceinline__ floatx4 multiply16(u32x4 a, u32x4 b, floatx4 c, __bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 multiply16(u32x4 a, u32x4 b, floatx4 c, float) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
  return c;
}

// Rows `first` .. of the expert, up to 16 NT of them.
template <typename T, int NT>
__device__ __forceinline__ void few_rows(const FewArgs& g, const T* x, const T* w, T* out, int64_t first, int64_t end,
                                         int64_t n0, floatx4 (*sums)[NT][64]) {
  constexpr int N = Vec<T>::N, kStep = 4 * N;  // k values of one step
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, kl = (lane >> 4) * N;
  // rows past the matrix and past the expert's are their last ones again: their outputs are not stored
  const T* pw = w + min(n0 + row, g.cols - 1) * g.ld_w + kl;
  const T* px[NT];
  bool none[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t r = min(first + 16 * n + row, end - 1), t = g.token.p ? g.token.get(r) : r;
    none[n] = t < 0 || t >= g.tokens;  // a row of zeros
    px[n] = x + (none[n] ? 0 : t * g.ld_x) + kl;
  }
  floatx4 s[NT] = {};
  // kAhead steps' loads are in flight at a time (2, 4, 8, 16 of them: 67.8, 65.7, 63.2, 149 us
  // for one row each of 64 experts of 1408 x 2048 in bfloat16, 369 MB, and for one row of 8 of
  // 2048 x 768 6.4, 7.4, 7.5, 11.0; with the weights read past the caches 72.5 and 7.5)
  constexpr int kAhead = 4;
  constexpr int64_t kStride = kFewWaves * kStep;
  int64_t k = (int64_t)wave * kStep;
  for (; k + (kAhead - 1) * kStride + kStep <= g.dim; k += kAhead * kStride) {
    u32x4 a[kAhead], c[kAhead][NT];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      a[i] = *reinterpret_cast<const u32x4_any*>(pw + k + i * kStride);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        c[i][n] = (u32x4){};
        if (!none[n]) c[i][n] = *reinterpret_cast<const u32x4_any*>(px[n] + k + i * kStride);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n] = multiply16(a[i], c[i][n], s[n], T());
  }
  for (; k < g.dim; k += kStride) {
    const int64_t left = g.dim - k - kl;
    const u32x4 a = load_raw<T>(pw + k, left);
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n] = multiply16(a, load_raw<T>(px[n] + k, none[n] ? 0 : left), s[n], T());
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) sums[wave][n][lane] = s[n];
  __syncthreads();
  // lane l holds columns n0 + 4 (l / 16) .. + 3 of row l % 16; wave n finishes 16 rows
  const int64_t r = first + 16 * wave + row;
  if (wave < NT && r < end) {
    floatx4 v = {};
    for (int i = 0; i < kFewWaves; ++i) v += sums[i][wave][lane];
    const int64_t col = n0 + 4 * (lane >> 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < g.cols) out[r * g.ld_out + col + e] = (T)v[e];
  }
  __syncthreads();  // the sums are read
}

template <typename T, int NT>
__global__ void __launch_bounds__(64 * kFewWaves, 4) expert_few_kernel(FewArgs g, const T* x, const T* w, T* out, int blocks_n) {
  __shared__ floatx4 sums[kFewWaves][NT][64];
  const int e = blockIdx.x / blocks_n;
  const int64_t n0 = (int64_t)(blockIdx.x - e * blocks_n) * 16;
  int64_t first, end;
  g.groups.rows_of(e, first, end);
  if (e == g.groups.experts) {  // rows of no expert: zeros
    for (int64_t i = threadIdx.x; i < (end - first) * 16; i += 64 * kFewWaves) {
      const int64_t col = n0 + (i & 15);
      if (col < g.cols) out[(first + (i >> 4)) * g.ld_out + col] = (T)0.f;
    }
    return;
  }
  w += e * g.stride_w;
  for (; first < end; first += 16 * NT) few_rows<T, NT>(g, x, w, out, first, end, n0, sums);
}

// Up to this many rows an expert, on average, come here, the others go to the tiles.  Both
// sides measured, us a call of a graph, here / tiles, for 64 experts of 1408 x 2048 and for 8 of
// 2048 x 768:
//   rows an expert   1             4             8             16            32            64            96
//   bfloat16         65.7 / 78.2   69.5 / 78.1   82.8 / 80.0   109 / 105     142 / 107     263 / 112
//                    7.4 / 12.1    8.2 / 12.5    8.9 / 12.5    10.9 / 13.8   12.9 / 13.0   22.2 / 13.5
//   float32          134 / 716     149 / 721     170 / 718     227 / 729     292 / 739     531 / 761     773 / 952
//                    13.9 / 50.0   14.2 / 49.2   14.5 / 49.5   20.3 / 50.1   23.4 / 51.4   40.8 / 55.0   58.2 / 60.9
// bfloat16 weights that the tiles would have copied first (150 us of the first kind) are as
// float32 in this.  The host knows the mean alone, and the rows above are spread as evenly as they
// can be: an expert that has most of them is walked by the workgroups of its columns, 16 or 32
// rows at a time, on a fraction of the card.
bool few_of(int32_t dtype, int64_t rows, int64_t experts, int64_t cols, bool copies) {
  return rows <= (dtype == ISOLOCO_F32 ? 96 : copies ? 48 : 16) * experts &&
         launchable((experts + 1) * ((cols + 15) / 16), 64 * kFewWaves);
}

template <typename T, int NT>
void launch_few_rows(const FewArgs& g, const void* x, const void* w, void* out, hipStream_t st) {
  const int blocks_n = (int)((g.cols + 15) / 16);
  hipLaunchKernelGGL((expert_few_kernel<T, NT>), dim3((unsigned)((g.groups.experts + 1) * blocks_n)), dim3(64 * kFewWaves), 0,
                     st, g, static_cast<const T*>(x), static_cast<const T*>(w), static_cast<T*>(out), blocks_n);
}

// 16 rows at a time, or 32 where an expert has more on average than 8: 16 rows each of 64 experts,
// as above, 106 / 109 us in bfloat16 and 209 / 227 in float32, 24 rows 186 / 125 and 351 / 258.
// (64 at a time: 24 rows 181 and 390.)
template <typename T>
hipError_t launch_few(const FewArgs& g, const void* x, const void* w, void* out, hipStream_t st) {
  if (g.groups.rows <= 8 * g.groups.experts) launch_few_rows<T, 1>(g, x, w, out, st);
  else launch_few_rows<T, 2>(g, x, w, out, st);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The tile products' operands
// ---------------------------------------------------------------------------

// What a call hands to the tile products, and where its copies lie in the workspace.
struct CallPlan {
  bool few;                     // expert_few_kernel
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
  p.few = !back && few_of(s.dtype, s.rows, s.experts, s.cols, !w_ok);
  if (p.few) return p;
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
  p.partial = take(back ? expert_gradients_partial_bytes(f32, s.rows, s.experts, s.dim, s.cols)
                        : expert_out_partial_bytes(f32, s.rows, s.experts, s.cols, s.dim));
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
  if (p.few) {
    const FewArgs g = {{c.offsets, c.s.rows, (int)c.s.experts}, c.token, c.s.tokens, c.s.dim, c.s.cols, c.ld_x, c.ld_w,
                       c.stride_w, ld_out};
    return c.s.dtype == ISOLOCO_F32 ? launch_few<float>(g, c.x, c.w, out, st) : launch_few<__bf16>(g, c.x, c.w, out, st);
  }
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
  return launch_expert_out(c.s.dtype == ISOLOCO_F32, g, st);
}

// wide_dx: dx of float32, past: and past the caches
hipError_t run_backward(const Call& c, const CallPlan& p, void* dx, int64_t ld_dx, bool wide_dx, bool past, void* dw, int64_t ld_dw,
                        int64_t stride_dw, char* ws, hipStream_t st) {
  const bool f32 = c.s.dtype == ISOLOCO_F32;
  const int64_t dim = ffn_pad(c.s.dim), cols = ffn_pad(c.s.cols);
  const Operands o = copy_operands(c, p, ws, st);
  ExpertArgs g = args_of(c, o, p, ws);
  g.a = o.d;
  g.ld_a = o.ld_d;
  g.part_a = o.part_d;
  g.n = c.s.dim;
  ExpertArgs x = g, w = g;
  x.token = {};
  x.b = o.w;
  x.ld_b = o.ld_w;
  x.part_b = o.part_w;
  x.stride_b = o.stride_w;
  x.cols_b = p.copy_w ? dim : c.s.dim;
  x.k = c.s.cols;
  x.out = dx;
  x.ld_out = ld_dx;
  x.wide_out = wide_dx;
  x.past = past;
  w.b = o.x;
  w.ld_b = o.ld_x;
  w.part_b = o.part_x;
  w.cols_a = p.copy_d ? cols : c.s.cols;
  w.cols_b = p.copy_x ? dim : c.s.dim;
  w.m = c.s.cols;
  w.out = dw;
  w.ld_out = ld_dw;
  w.stride_out = stride_dw;
  return launch_expert_gradients(f32, dx ? &x : nullptr, dw ? &w : nullptr, st);
}

// What a call of the gradients is given.
struct Gradients {
  ExpertShape s;
  const void *x, *token, *w, *offsets, *dout;
  int64_t ld_x, ld_w, stride_w, ld_dout;
  int32_t index_type;
  void *dx, *dw;
  int64_t ld_dx, ld_dw, stride_dw;
  // dx of the tokens: the sums of float32 rows, which are formed in dx_rows
  const void* row;
  int32_t row_type, top_k;
  float* dx_rows;
  bool sum;
};

isoloco_status gradients(Gradients g, void* workspace, size_t workspace_bytes, hipStream_t st) {
  const ExpertShape& s = g.s;
  ISOLOCO_TRY(check_shape(s));
  if (!is_index_type(g.index_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type %d", g.index_type);
  if (!g.token && !g.sum && s.rows && s.tokens != s.rows)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of x, %lld wanted", (long long)s.tokens, (long long)s.rows);
  const size_t e = dtype_bytes(s.dtype), ib = index_bytes(g.index_type);
  if (g.sum) {
    if (!is_index_type(g.row_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type of row %d", g.row_type);
    if (g.top_k < 1 || g.top_k > ISOLOCO_MAX_TOP)
      return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d, of 1 to %d", g.top_k, ISOLOCO_MAX_TOP);
  }
  const int64_t dx_rows = g.sum ? s.tokens : s.rows;
  const bool dx = (g.dx || g.sum) && dx_rows;
  if (!dx && !g.dw) return ISOLOCO_OK;
  if (g.dw) {
    ISOLOCO_TRY(check_matrix("x", g.x, s.tokens, s.dim, g.ld_x, e));
    ISOLOCO_TRY(check_experts("dw", g.dw, s, g.ld_dw, g.stride_dw));
  }
  if (dx && s.rows) ISOLOCO_TRY(check_experts("w", g.w, s, g.ld_w, g.stride_w));
  if (dx) ISOLOCO_TRY(check_matrix("dx", g.dx, dx_rows, s.dim, g.ld_dx, e));
  ISOLOCO_TRY(check_matrix("dout", g.dout, s.rows, s.cols, g.ld_dout, e));
  void* rows_out = !dx || s.rows == 0 ? nullptr : g.sum ? static_cast<void*>(g.dx_rows) : g.dx;
  // (no rows and no dw: nothing to multiply, and dx of the tokens is zeros)
  const bool products = rows_out || g.dw;
  CallPlan p = {};
  if (products)
    p = call_plan(s, g.token, rows_out, g.dw, tile_rows(g.x, s.dim, g.ld_x),
                  tile_rows(g.w, s.dim, g.ld_w) && (s.experts == 1 || (g.stride_w & 7) == 0),
                  tile_rows(g.dout, s.cols, g.ld_dout), g.ld_x);
  const size_t need = p.bytes;
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const size_t row_bytes = g.sum ? (size_t)s.tokens * g.top_k * index_bytes(g.row_type) : 0;
  const Operand ins[] = {{"x", g.x, g.dw ? matrix_bytes(s.tokens, s.dim, g.ld_x, e) : 0, e},
                         {"w", g.w, dx && s.rows ? experts_bytes(s, g.ld_w, g.stride_w) : 0, e},
                         {"dout", g.dout, matrix_bytes(s.rows, s.cols, g.ld_dout, e), e},
                         {"offsets", g.offsets, (size_t)(s.experts + 1) * ib, ib},
                         {"token", g.token, g.sum || (g.token && g.dw) ? (size_t)s.rows * ib : 0, ib},
                         {"row", g.row, row_bytes, g.sum ? index_bytes(g.row_type) : 1}};
  const Operand outs[] = {{"dx", g.dx, dx ? matrix_bytes(dx_rows, s.dim, g.ld_dx, e) : 0, e},
                          {"dw", g.dw, g.dw ? experts_bytes(s, g.ld_dw, g.stride_dw) : 0, e},
                          {"the workspace", workspace, need, 1},
                          {"dx_rows", g.dx_rows, g.sum ? (size_t)s.rows * s.dim * 4 : 0, 4}};
  ISOLOCO_TRY(check_operands(outs, 4, ins, 6));
  const bool wide = g.index_type == ISOLOCO_I64;
  const Call c = {s, g.x, g.w, g.dout, g.ld_x, g.ld_w, g.stride_w, g.ld_dout, {g.offsets, wide}, {g.token, wide}};
  // (both passes over 131072 rows of 2048 of them, past the caches / through them: 1034 / 1090 us)
  const bool past = g.sum && s.dtype == ISOLOCO_BF16 && s.rows * s.dim * 4 > kCacheBytes;
  hipError_t r = hipSuccess;
  if (products)
    r = run_backward(c, p, rows_out, g.sum ? s.dim : g.ld_dx, g.sum, past, g.dw, g.ld_dw, g.stride_dw,
                     static_cast<char*>(workspace), st);
  if (r == hipSuccess && g.sum)
    r = launch_rows_sum(g.dx_rows, s.rows, s.dim, {g.row, g.row_type == ISOLOCO_I64}, s.tokens, g.top_k,
                        s.dtype == ISOLOCO_F32, past, g.dx, g.ld_dx, st);
  return r == hipSuccess ? ISOLOCO_OK : hip_fail(r, "gradient of products grouped by expert");
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
  // (without ALIGNED each operand may be either)
  const bool gathered = flags & ISOLOCO_EXPERTS_GATHERED;
  *bytes = 0;
  for (int i = ok ? 7 : 0; i < 8; ++i)
    *bytes = std::max(*bytes, call_plan(s, gathered, back, back, i & 1, i & 2, i & 4, ld_x).bytes);
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
  if (!token && rows && tokens != rows) return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of x, %lld wanted", (long long)tokens, (long long)rows);
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
  Gradients g = {};
  g.s = {tokens, rows, experts, dim, cols, dtype};
  g.x = x, g.token = token, g.w = w, g.offsets = offsets, g.dout = dout;
  g.ld_x = ld_x, g.ld_w = ld_w, g.stride_w = stride_w, g.ld_dout = ld_dout;
  g.index_type = index_type;
  g.dx = dx, g.dw = dw;
  g.ld_dx = ld_dx, g.ld_dw = ld_dw, g.stride_dw = stride_dw;
  return gradients(g, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}

isoloco_status isoloco_expert_matmul_backward_tokens(const void* x, int64_t ld_x, int64_t tokens, const void* token,
                                                     const void* row, int32_t row_type, int32_t top_k, const void* w,
                                                     int64_t ld_w, int64_t stride_w, int32_t dtype, const void* offsets,
                                                     int32_t index_type, int64_t experts, int64_t rows, int64_t dim,
                                                     int64_t cols, const void* dout, int64_t ld_dout, void* dx,
                                                     int64_t ld_dx, float* dx_rows, void* dw, int64_t ld_dw,
                                                     int64_t stride_dw, void* workspace, size_t workspace_bytes,
                                                     void* hip_stream) {
  Gradients g = {};
  g.s = {tokens, rows, experts, dim, cols, dtype};
  g.x = x, g.token = token, g.w = w, g.offsets = offsets, g.dout = dout;
  g.ld_x = ld_x, g.ld_w = ld_w, g.stride_w = stride_w, g.ld_dout = ld_dout;
  g.index_type = index_type;
  g.dx = dx, g.dw = dw;
  g.ld_dx = ld_dx, g.ld_dw = ld_dw, g.stride_dw = stride_dw;
  g.row = row, g.row_type = row_type, g.top_k = top_k;
  g.dx_rows = dx_rows;
  g.sum = true;
  return gradients(g, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
