// The sum of a token's rows, as they come back from the experts:
//
//   out[t] = sum_j weight[t, j] y[row[t, j]]
//   dy[row[t, j]] = weight[t, j] dout[t],   dweight[t, j] = <dout[t], y[row[t, j]]>
//   (zeros in rows that no slot names)
//
// The terms of a sum are added in the order of j; no two slots name one row, so that
// nothing is added across tokens.  Bounded by memory: every row is read once (backward:
// and its gradient written once).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_experts.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

struct CombineArgs {
  Index row;
  const float* weight;  // or NULL: ones
  int64_t tokens, rows, dim, ld_y, ld_out;
  int top_k;
};

constexpr int kAtOnce = 8;  // rows whose pieces a thread has in flight

// One thread per piece of 16 bytes of y's rows (16384 tokens of 8 rows of 2048 in bfloat16:
// 120 us, 5.0 TB/s; with the rows read past the caches 27 us more).  PAST: of rows that were
// stored past the caches.
template <typename T, typename O, bool PAST>
__global__ void __launch_bounds__(256) combine_kernel(const T* y, O* out, CombineArgs g, int pieces) {
  constexpr int N = Vec<T>::N;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x, t = item / pieces;
  if (t >= g.tokens) return;
  const int64_t col = (item - t * pieces) * N, left = g.dim - col;
  float sum[N] = {};
  for (int j0 = 0; j0 < g.top_k; j0 += kAtOnce) {
    u32x4 v[kAtOnce];
    float w[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int j = j0 + u;
      const int64_t r = j < g.top_k ? g.row.get(t * g.top_k + j) : -1;
      const bool in = r >= 0 && r < g.rows;
      w[u] = in ? (g.weight ? g.weight[t * g.top_k + j] : 1.f) : 0.f;
      v[u] = (u32x4){};
      if (in) v[u] = load_raw<T, PAST>(y + r * g.ld_y + col, left);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      float x[N];
      unpack<T>(v[u], x);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] = fmaf(w[u], x[e], sum[e]);
    }
  }
  O* to = out + t * g.ld_out + col;
  if constexpr (sizeof(O) == sizeof(T)) {
    store_piece<O>(to, left, sum);
  } else if (left >= N) {
    // (half a piece)
    *reinterpret_cast<u32x2_any*>(to) = pack4(sum);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) to[e] = (O)sum[e];
  }
}

// Rows of dy that no slot names have no gradient, and are cleared before the named rows are written
// (clearing all of them costs 105 us of 344 for 537 MB).  Where there are as many slots as rows or
// more, the rows that slots name are marked, a bit each: by every workgroup that clears, if the
// slots are few, otherwise ahead of it, where each workgroup finds the slots of its rows among all
// (131072 slots: 9.6 us, 11.7 with a load a slot, and the clearing that finds none to clear 4.5).
// Counting the slots takes half of it, but tells nothing where two name one row and leave another
// without any.
constexpr int64_t kFewSlots = 8192;
constexpr int kMarkThreads = 1024;
constexpr int64_t kMostMarked = (int64_t)1 << 18;  // rows of a workgroup that marks: 32 KiB of bits

// The bits of rows first .. first + count - 1, in `bits`, by the workgroup.
template <typename ID, int THREADS>
__device__ __forceinline__ void mark_rows(const ID* row, int64_t slots, int64_t first, int64_t count, uint32_t* bits) {
  typedef typename std::make_unsigned<ID>::type U;
  for (int64_t i = threadIdx.x; i < (count + 31) / 32; i += THREADS) bits[i] = 0;
  __syncthreads();
  const U from = (U)first, many = (U)count;
  const auto mark = [&](ID at) {
    const U r = (U)at - from;
    if (r < many) atomicOr(&bits[(uint32_t)r >> 5], 1u << ((uint32_t)r & 31));
  };
  // 16 bytes of slots a load, and so many loads in flight
  constexpr int kPer = 16 / sizeof(ID), kAhead = 8;
  int64_t base = 0;
  for (; base + kPer * kAhead * THREADS <= slots; base += kPer * kAhead * THREADS) {
    const u32x4_any* p = reinterpret_cast<const u32x4_any*>(row + base);
    u32x4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = p[u * THREADS + (int)threadIdx.x];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      ID r[kPer];
      __builtin_memcpy(r, &v[u], 16);
#pragma unroll
      for (int e = 0; e < kPer; ++e) mark(r[e]);
    }
  }
  for (int64_t i = base + threadIdx.x; i < slots; i += THREADS) mark(row[i]);
  __syncthreads();
}
template <int THREADS>
__device__ __forceinline__ void mark_rows(const Index& row, int64_t slots, int64_t first, int64_t count, uint32_t* bits) {
  if (row.wide) mark_rows<int64_t, THREADS>(static_cast<const int64_t*>(row.p), slots, first, count, bits);
  else mark_rows<int32_t, THREADS>(static_cast<const int32_t*>(row.p), slots, first, count, bits);
}

// per: rows of a workgroup, a multiple of 32
__global__ void __launch_bounds__(kMarkThreads) combine_mark_kernel(Index row, int64_t rows, int64_t slots, int64_t per,
                                                                    uint32_t* marks) {
  __shared__ uint32_t bits[kMostMarked / 32];
  const int64_t first = blockIdx.x * per, count = min(per, rows - first);
  mark_rows<kMarkThreads>(row, slots, first, count, bits);
  for (int64_t i = threadIdx.x; i < (count + 31) / 32; i += kMarkThreads) marks[first / 32 + i] = bits[i];
}

// MARKED: the rows' bits are in `marks`, FEW: they are formed here, ALL: no row is marked.
enum Clearing { kMarked, kFew, kAll };
template <typename T, Clearing HOW>
__global__ void __launch_bounds__(256) combine_clear_kernel(Index row, int64_t rows, int64_t slots, const uint32_t* marks,
                                                            T* dy, int64_t ld, int64_t dim) {
  __shared__ uint32_t bits[HOW == kFew ? kFewSlots / 32 : 1];
  if constexpr (HOW == kFew) mark_rows<256>(row, slots, 0, rows, bits);
  constexpr int N = Vec<T>::N;
  const float zeros[N] = {};
  const int64_t pieces = (dim + N - 1) / N, words = (rows + 31) / 32, from = words * blockIdx.x / gridDim.x, to = words * (blockIdx.x + 1) / gridDim.x;
  for (int64_t w = from; w < to; ++w) {
    uint32_t none = ~(HOW == kAll ? 0u : HOW == kFew ? bits[w] : marks[w]);
    if (rows - 32 * w < 32) none &= (1u << (rows - 32 * w)) - 1;
    if (none == 0) continue;
    for (int64_t i = (int64_t)blockIdx.y * 256 + threadIdx.x; i < 32 * pieces; i += (int64_t)gridDim.y * 256) {
      const int64_t r = i / pieces, col = (i - r * pieces) * N;
      if (none >> r & 1u) store_piece<T>(dy + (32 * w + r) * ld + col, dim - col, zeros);
    }
  }
}

struct CombineGradArgs {
  Index row;
  const float* weight;
  int64_t tokens, rows, dim, ld_dout, ld_y, ld_dy;
  int top_k;
  float* dweight;
  int lanes_log2;  // threads of a token: 2^this
};

// 2^lanes_log2 threads per token, which go through its columns kAtOnce slots at a time.  The
// pieces stay as they are stored until they are used, and the stores go ahead of the products:
// 16384 tokens of 8 rows of 2048 in bfloat16 take 222 us (1141 MB, 5.1 TB/s) where unpacked
// ones took 326.  64 / 128 / 256 threads a token: both passes 363 / 357 / 364 us.
constexpr int kMostLanesLog2 = 7;

// PAST: y and its gradient go past the caches.
template <typename T, bool DY, bool DW, bool PAST>
__global__ void __launch_bounds__(256) combine_grad_kernel(const T* dout, const T* y, T* dy, CombineGradArgs g) {
  constexpr int N = Vec<T>::N;
  __shared__ float part[4][kAtOnce];
  const int lanes = 1 << g.lanes_log2, in = threadIdx.x & (lanes - 1);
  const int64_t t = ((int64_t)blockIdx.x << (8 - g.lanes_log2)) + (threadIdx.x >> g.lanes_log2);
  const bool live = t < g.tokens;
  const T* d = dout + t * g.ld_dout;
  for (int j0 = 0; j0 < g.top_k; j0 += kAtOnce) {
    int64_t r[kAtOnce];
    float w[kAtOnce], dot[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int j = j0 + u;
      r[u] = live && j < g.top_k ? g.row.get(t * g.top_k + j) : -1;
      if (r[u] >= g.rows) r[u] = -1;
      w[u] = r[u] >= 0 && g.weight ? g.weight[t * g.top_k + j] : 1.f;
      dot[u] = 0.f;
    }
    if (live) {
      for (int64_t col = (int64_t)in * N; col < g.dim; col += (int64_t)lanes * N) {
        const int64_t left = g.dim - col;
        float a[N];
        u32x4 v[kAtOnce];
        load_piece<T>(d + col, left, a);
        if constexpr (DW) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            v[u] = (u32x4){};
            if (r[u] >= 0) v[u] = load_raw<T, PAST>(y + r[u] * g.ld_y + col, left);
          }
        }
        if constexpr (DY) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = w[u] * a[e];
            if (r[u] >= 0) store_piece<T, PAST>(dy + r[u] * g.ld_dy + col, left, x);
          }
        }
        if constexpr (DW) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            float x[N];
            unpack<T>(v[u], x);
#pragma unroll
            for (int e = 0; e < N; ++e)
              if (r[u] >= 0) dot[u] = fmaf(a[e], x[e], dot[u]);
          }
        }
      }
    }
    if constexpr (DW) {
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        for (int off = std::min(lanes, 64) >> 1; off > 0; off >>= 1) dot[u] += __shfl_xor(dot[u], off, 64);
      if (lanes > 64) {
        const int wave = threadIdx.x >> 6, waves = lanes >> 6, first = wave & ~(waves - 1);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) part[wave][u] = dot[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          dot[u] = part[first][u];
          for (int v = 1; v < waves; ++v) dot[u] += part[first + v][u];
        }
      }
      if (live && in == 0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
          if (j0 + u < g.top_k) g.dweight[t * g.top_k + j0 + u] = dot[u];
      }
    }
  }
}

template <typename T, typename O = T, bool PAST = false>
void run_forward(const void* y, void* out, const CombineArgs& g, int pieces, int64_t blocks, hipStream_t st) {
  hipLaunchKernelGGL((combine_kernel<T, O, PAST>), dim3((unsigned)blocks), dim3(256), 0, st, static_cast<const T*>(y),
                     static_cast<O*>(out), g, pieces);
}

// the marks of as many rows as slots
size_t combine_grad_workspace(int64_t tokens, int32_t top_k) {
  const int64_t slots = tokens * top_k;
  return slots > kFewSlots ? (size_t)(slots + 31) / 32 * sizeof(uint32_t) : 0;
}

template <typename T>
void clear_rows(const CombineGradArgs& g, T* dy, uint32_t* marks, hipStream_t st) {
  const int64_t slots = g.tokens * g.top_k, rows = g.rows;
  // about 1024 workgroups; where the rows are fewer than those take, some share 32 rows
  const int64_t words = (rows + 31) / 32, pieces = (g.dim + Vec<T>::N - 1) / Vec<T>::N;
  const dim3 grid((unsigned)std::min<int64_t>(1024, words),
                  (unsigned)std::min(std::max<int64_t>(1, 1024 / words), (pieces + 31) / 32));
  if (rows > slots) {
    hipLaunchKernelGGL((combine_clear_kernel<T, kAll>), grid, dim3(256), 0, st, g.row, rows, slots, marks, dy, g.ld_dy, g.dim);
  } else if (slots <= kFewSlots) {
    hipLaunchKernelGGL((combine_clear_kernel<T, kFew>), grid, dim3(256), 0, st, g.row, rows, slots, marks, dy, g.ld_dy, g.dim);
  } else {
    // about a workgroup a CU
    const int64_t per = std::min(kMostMarked, (rows / 256 / 32 + 1) * 32);
    hipLaunchKernelGGL(combine_mark_kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(kMarkThreads), 0, st, g.row, rows,
                       slots, per, marks);
    hipLaunchKernelGGL((combine_clear_kernel<T, kMarked>), grid, dim3(256), 0, st, g.row, rows, slots, marks, dy, g.ld_dy,
                       g.dim);
  }
}

template <typename T, bool PAST>
void run_grad(const void* dout, const void* y, void* dy, const CombineGradArgs& g, int64_t blocks, uint32_t* marks,
              hipStream_t st) {
  if (dy && g.rows) clear_rows(g, static_cast<T*>(dy), marks, st);
  if (blocks == 0) return;
  const dim3 grid((unsigned)blocks);
  const T *d = static_cast<const T*>(dout), *x = static_cast<const T*>(y);
  T* o = static_cast<T*>(dy);
  if (dy && g.dweight) hipLaunchKernelGGL((combine_grad_kernel<T, true, true, PAST>), grid, dim3(256), 0, st, d, x, o, g);
  else if (dy) hipLaunchKernelGGL((combine_grad_kernel<T, true, false, PAST>), grid, dim3(256), 0, st, d, x, o, g);
  else hipLaunchKernelGGL((combine_grad_kernel<T, false, true, PAST>), grid, dim3(256), 0, st, d, x, o, g);
}

isoloco_status check_shape(int32_t dtype, int64_t tokens, int64_t rows, int64_t dim, int32_t index_type, int32_t top_k) {
  if (tokens < 0 || tokens > kMaxExtent / 2 || rows < 0 || rows > kMaxExtent || dim < 1 || dim > kMaxExtent / 2)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld tokens of %lld rows, dim %lld", (long long)tokens, (long long)rows,
                (long long)dim);
  if (top_k < 1 || top_k > ISOLOCO_MAX_TOP)
    return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d, of 1 to %d", top_k, ISOLOCO_MAX_TOP);
  if (!is_dtype(dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", dtype);
  if (!is_index_type(index_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type %d", index_type);
  return ISOLOCO_OK;
}

}  // namespace

hipError_t launch_rows_sum(const float* y, int64_t rows, int64_t dim, Index row, int64_t tokens, int top_k, bool f32,
                           bool past, void* out, int64_t ld_out, hipStream_t st) {
  // so many tokens as one launch has threads for
  const int64_t pieces = (dim + 3) / 4, most = ((int64_t)1 << 31) / pieces;
  const int64_t row_bytes = (int64_t)top_k * (row.wide ? 8 : 4), out_bytes = ld_out * (f32 ? 4 : 2);
  for (int64_t t = 0; t < tokens; t += most) {
    const CombineArgs g = {{static_cast<const char*>(row.p) + t * row_bytes, row.wide}, nullptr, std::min(most, tokens - t), rows,
                           dim, dim, ld_out, top_k};
    const int64_t blocks = (g.tokens * pieces + 255) / 256;
    void* to = static_cast<char*>(out) + t * out_bytes;
    if (f32) run_forward<float>(y, to, g, (int)pieces, blocks, st);
    else if (past) run_forward<float, __bf16, true>(y, to, g, (int)pieces, blocks, st);
    else run_forward<float, __bf16>(y, to, g, (int)pieces, blocks, st);
  }
  return hipGetLastError();
}

}  // namespace isoloco

using namespace isoloco;

extern "C" {

isoloco_status isoloco_combine_tokens(const void* y, int64_t ld_y, int32_t dtype, int64_t rows, int64_t dim,
                                      const void* row, int32_t index_type, const float* weight, int64_t tokens,
                                      int32_t top_k, void* out, int64_t ld_out, void* hip_stream) {
  ISOLOCO_TRY(check_shape(dtype, tokens, rows, dim, index_type, top_k));
  if (tokens == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type), n = (size_t)tokens * top_k;
  ISOLOCO_TRY(check_matrix("y", y, rows, dim, ld_y, e));
  ISOLOCO_TRY(check_matrix("out", out, tokens, dim, ld_out, e));
  const Operand ins[] = {{"y", y, matrix_bytes(rows, dim, ld_y, e), e},
                         {"row", row, n * ib, ib},
                         {"weight", weight, weight ? n * 4 : 0, 4}};
  const Operand outs[] = {{"out", out, matrix_bytes(tokens, dim, ld_out, e), e}};
  ISOLOCO_TRY(check_operands(outs, 1, ins, 3));
  const int64_t per = 16 / (int64_t)e, pieces = (dim + per - 1) / per, blocks = (tokens * pieces + 255) / 256;
  if (!launchable(blocks, 256)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  const CombineArgs g = {{row, index_type == ISOLOCO_I64}, weight, tokens, rows, dim, ld_y, ld_out, top_k};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == ISOLOCO_F32) run_forward<float>(y, out, g, (int)pieces, blocks, st);
  else run_forward<__bf16>(y, out, g, (int)pieces, blocks, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "combination of tokens");
}

isoloco_status isoloco_combine_tokens_backward_workspace_size(int64_t tokens, int32_t top_k, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  ISOLOCO_TRY(check_shape(ISOLOCO_F32, tokens, 0, 1, ISOLOCO_I32, top_k));
  *bytes = combine_grad_workspace(tokens, top_k);
  return ISOLOCO_OK;
}

isoloco_status isoloco_combine_tokens_backward(const void* dout, int64_t ld_dout, const void* y, int64_t ld_y,
                                               int32_t dtype, int64_t rows, int64_t dim, const void* row,
                                               int32_t index_type, const float* weight, int64_t tokens, int32_t top_k,
                                               void* dy, int64_t ld_dy, float* dweight, void* workspace,
                                               size_t workspace_bytes, void* hip_stream) {
  ISOLOCO_TRY(check_shape(dtype, tokens, rows, dim, index_type, top_k));
  if (dweight && !weight) return fail(ISOLOCO_ERR_INVALID_ARG, "dweight needs weight");
  if (!dy && !dweight) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type), n = (size_t)tokens * top_k;
  const size_t need = dy ? combine_grad_workspace(tokens, top_k) : 0;
  ISOLOCO_TRY(check_matrix("dout", dout, tokens, dim, ld_dout, e));
  if (dweight) ISOLOCO_TRY(check_matrix("y", y, rows, dim, ld_y, e));
  if (dy) ISOLOCO_TRY(check_matrix("dy", dy, rows, dim, ld_dy, e));
  const Operand ins[] = {{"dout", dout, matrix_bytes(tokens, dim, ld_dout, e), e},
                         {"y", y, dweight ? matrix_bytes(rows, dim, ld_y, e) : 0, e},
                         {"row", row, n * ib, ib},
                         {"weight", weight, weight ? n * 4 : 0, 4}};
  const Operand outs[] = {{"dy", dy, dy ? matrix_bytes(rows, dim, ld_dy, e) : 0, e},
                          {"dweight", dweight, dweight ? n * 4 : 0, 4},
                          {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  ISOLOCO_TRY(check_operands(outs, 3, ins, 4));
  CombineGradArgs g = {{row, index_type == ISOLOCO_I64}, weight, tokens, rows, dim, ld_dout, ld_y, ld_dy, top_k, dweight, 3};
  const int64_t per = 16 / (int64_t)e;
  while (g.lanes_log2 < kMostLanesLog2 && (per << g.lanes_log2) < dim) ++g.lanes_log2;
  const int64_t blocks = (tokens + (256 >> g.lanes_log2) - 1) >> (8 - g.lanes_log2);
  if (!launchable(blocks, 256)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many tokens for one launch");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  uint32_t* marks = static_cast<uint32_t*>(workspace);
  // Both sides measured, past the caches / through them, us of both passes over 537 MB of rows:
  // 357 / 379.
  const bool past = rows * dim * (int64_t)e > kCacheBytes;
  if (dtype == ISOLOCO_F32) (past ? run_grad<float, true> : run_grad<float, false>)(dout, y, dy, g, blocks, marks, st);
  else (past ? run_grad<__bf16, true> : run_grad<__bf16, false>)(dout, y, dy, g, blocks, marks, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "gradient of the combination of tokens");
}

}  // extern "C"
