// The global norm of many tensors, and clipping by it.
//
//   norm = sqrt(sum over every tensor and element of g^2)
//   coef = max_norm / norm if max_norm < norm < infinity, else 1;   dst = coef * g
//
// Two passes over the data: the norm has to be known before the first scaled
// value is written.  Bounded by memory: the norm reads every byte once, the
// scaling reads and writes it.
#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "isoloco_device.h"
#include "isoloco_error.h"

namespace isoloco {
namespace {

// Tensors per launch: their pointers and sizes travel in the launch's arguments
// (3.9 of the 4 KiB that these may take), so that no table is copied to the device.
constexpr int kClipTensors = 160;
constexpr int kClipThreads = 512;
// Four workgroups of 8 waves fill a CU.  The number of partial sums of a launch.
constexpr int kClipBlocks = 1024;
constexpr int kVecBytes = 16, kUnroll = 4;
// The unit of work: what a workgroup loads at once.
constexpr int kChunkBytes = kClipThreads * kVecBytes * kUnroll;

struct ClipArgs {
  const void* src[kClipTensors];
  void* dst[kClipTensors];
  int32_t first[kClipTensors + 1];  // first chunk of each tensor; then the number of chunks
  int32_t last[kClipTensors];       // bytes of its last chunk (the others are whole)
  uint8_t bf16[kClipTensors];
  int32_t n;
  int32_t in_place;  // all of them
};

// 16 bytes at the alignment of an element: a tensor may start anywhere in a flat
// buffer (the hardware takes such accesses whole).
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// The tensor of a chunk (wave-uniform).
__device__ __forceinline__ int tensor_of(const ClipArgs& a, int chunk) {
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int chunk_bytes(const ClipArgs& a, int t, int chunk) {
  return chunk + 1 == a.first[t + 1] ? a.last[t] : kChunkBytes;
}

// Squares are summed in 64 bits: those of values past 1.8e19 or below 1e-23 leave
// the range of 32.
template <bool BF16>
__device__ __forceinline__ void add_squares(double& s, u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      const double lo = bf16_to_f32(v[i] & 0xffffu), hi = __uint_as_float(v[i] & 0xffff0000u);
      s = fma(lo, lo, s);
      s = fma(hi, hi, s);
    } else {
      const double x = __uint_as_float(v[i]);
      s = fma(x, x, s);
    }
  }
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const char* p, int bytes) {
  constexpr int kElem = BF16 ? 2 : 4;
  double s = 0.0;
  if (bytes >= kChunkBytes) {
    u32x4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      v[u] = *reinterpret_cast<const u32x4_any*>(p + (u * kClipThreads + (int)threadIdx.x) * kVecBytes);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) add_squares<BF16>(s, v[u]);
    return s;
  }
  const int whole = bytes / kVecBytes;
  for (int i = threadIdx.x; i < whole; i += kClipThreads)
    add_squares<BF16>(s, *reinterpret_cast<const u32x4_any*>(p + i * kVecBytes));
  const int at = whole * kVecBytes + (int)threadIdx.x * kElem;
  if (at < bytes) {
    const double x = BF16 ? (double)bf16_to_f32(*reinterpret_cast<const uint16_t*>(p + at))
                          : (double)*reinterpret_cast<const float*>(p + at);
    s = fma(x, x, s);
  }
  return s;
}

// Partial sums in a fixed order: which chunks a workgroup takes depends on the
// sizes alone.
__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(ClipArgs a, double* part) {
  __shared__ double lds[kClipThreads / 64];
  double s = 0.0;
  const int chunks = a.first[a.n];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = tensor_of(a, c);
    const char* p = static_cast<const char*>(a.src[t]) + (int64_t)(c - a.first[t]) * kChunkBytes;
    const int bytes = chunk_bytes(a, t, c);
    s += a.bf16[t] ? chunk_squares<true>(p, bytes) : chunk_squares<false>(p, bytes);
  }
  s = block_sum<kClipThreads / 64>(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// A coefficient as two factors, taken one after the other: below 2^-126 it has fewer
// bits in float32, or none, while its product with a large gradient has them all.  (The
// first of them is 2^-126 there and 1 otherwise; what it takes from a value the product
// has no place for either.)
struct Coef {
  float pre, c;
  __device__ __forceinline__ float of(float x) const { return x * pre * c; }
};

// The norm and the coefficient from the n partial sums of every launch, on every
// thread of a workgroup.
template <int WAVES>
__device__ __forceinline__ floatx2 norm_and_coef(const double* part, int n, float max_norm, double* lds, Coef& k) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += WAVES * 64) s += part[i];
  s = block_sum<WAVES>(s, lds);
  if (threadIdx.x == 0) lds[0] = s;
  __syncthreads();
  const double norm = sqrt(lds[0]);
  const double coef = norm > (double)max_norm && norm < (double)INFINITY ? (double)max_norm / norm : 1.0;
  const bool small = coef < (double)FLT_MIN;
  k = {small ? FLT_MIN : 1.f, (float)(small ? coef / (double)FLT_MIN : coef)};
  return (floatx2){(float)norm, (float)coef};
}

__global__ void __launch_bounds__(256) clip_finish_kernel(const double* part, int n, float max_norm, float* out) {
  __shared__ double lds[4];
  Coef k;
  const floatx2 r = norm_and_coef<4>(part, n, max_norm, lds, k);
  if (threadIdx.x == 0) {
    out[0] = r[0];
    out[1] = r[1];
  }
}

__device__ __forceinline__ uint32_t scale_pair(uint32_t v, Coef k) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t r = __builtin_convertvector((floatx2){k.of(bf16_to_f32(v & 0xffffu)), k.of(__uint_as_float(v & 0xffff0000u))},
                                             bf16x2_t);
  return __builtin_bit_cast(uint32_t, r);
}

template <bool BF16>
__device__ __forceinline__ u32x4 scaled(u32x4 v, Coef k) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = BF16 ? scale_pair(v[i], k) : __float_as_uint(k.of(__uint_as_float(v[i])));
  return v;
}

template <bool BF16>
__device__ __forceinline__ void scale_part(const char* p, char* q, int bytes, Coef k) {
  constexpr int kElem = BF16 ? 2 : 4;
  const int whole = bytes / kVecBytes;
  for (int i = threadIdx.x; i < whole; i += kClipThreads)
    *reinterpret_cast<u32x4_any*>(q + i * kVecBytes) =
        scaled<BF16>(*reinterpret_cast<const u32x4_any*>(p + i * kVecBytes), k);
  const int at = whole * kVecBytes + (int)threadIdx.x * kElem;
  if (at < bytes) {
    if constexpr (BF16)
      *reinterpret_cast<uint16_t*>(q + at) = (uint16_t)scale_pair(*reinterpret_cast<const uint16_t*>(p + at), k);
    else
      *reinterpret_cast<float*>(q + at) = k.of(*reinterpret_cast<const float*>(p + at));
  }
}

// Every workgroup forms the norm from the partial sums itself (a few KiB, read from the
// cache, while its first chunk is on its way) rather than wait for a launch that does it
// once.  (The chunk waits for the norm in place, where one below the bound leaves
// nothing to do.)  The last chunks go first: the norm's pass read them last, some are
// still in a cache.  PAST: results go past the caches.
template <bool PAST>
__global__ void __launch_bounds__(kClipThreads) clip_scale_kernel(ClipArgs a, const double* part, int n_part,
                                                                 float max_norm, float* out) {
  __shared__ double lds[kClipThreads / 64];
  Coef k = {0.f, 0.f};
  bool first = true;
  for (int c = a.first[a.n] - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const int t = tensor_of(a, c);
    const int64_t off = (int64_t)(c - a.first[t]) * kChunkBytes;
    const char* p = static_cast<const char*>(a.src[t]) + off;
    char* q = static_cast<char*>(a.dst[t]) + off;
    const int bytes = chunk_bytes(a, t, c);
    u32x4 v[kUnroll];
    const auto load = [&] {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        v[u] = *reinterpret_cast<const u32x4_any*>(p + (u * kClipThreads + (int)threadIdx.x) * kVecBytes);
    };
    const bool whole = bytes == kChunkBytes;
    if (first) {
      if (whole && !a.in_place) load();
      const floatx2 r = norm_and_coef<kClipThreads / 64>(part, n_part, max_norm, lds, k);
      if (out && blockIdx.x == 0 && threadIdx.x == 0) {
        out[0] = r[0];
        out[1] = r[1];
      }
      if (k.of(1.f) == 1.f && a.in_place) return;
    }
    // (coef 1 in place: the tensor stays as it is)
    if (p != q || k.of(1.f) != 1.f) {
      if (whole) {
        if (!first || a.in_place) load();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          u32x4_any* to = reinterpret_cast<u32x4_any*>(q + (u * kClipThreads + (int)threadIdx.x) * kVecBytes);
          const u32x4 r = a.bf16[t] ? scaled<true>(v[u], k) : scaled<false>(v[u], k);
          if constexpr (PAST) __builtin_nontemporal_store(r, to);
          else *to = r;
        }
      } else if (a.bf16[t]) {
        scale_part<true>(p, q, bytes, k);
      } else {
        scale_part<false>(p, q, bytes, k);
      }
    }
    first = false;
  }
}

size_t clip_workspace(int32_t n_tensors) {
  const size_t launches = ((size_t)n_tensors + kClipTensors - 1) / kClipTensors;
  return (launches ? launches : 1) * kClipBlocks * sizeof(double);
}

// No result overlaps another tensor or its result: workgroups take the tensors in no
// order.
isoloco_status check_results_apart(const void* const* src, void* const* dst, const int64_t* counts,
                                   const int32_t* dtypes, int32_t n_tensors) {
  struct Range {
    uintptr_t from, to;
    int32_t tensor;
    bool result;
  };
  const std::unique_ptr<Range[]> r(new (std::nothrow) Range[2 * (size_t)n_tensors]);
  if (!r) return fail(ISOLOCO_ERR_UNSUPPORTED, "no memory to check %d tensors", n_tensors);
  size_t n = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const uintptr_t bytes = (uintptr_t)counts[i] * dtype_bytes(dtypes[i]);
    const uintptr_t s = reinterpret_cast<uintptr_t>(src[i]), d = reinterpret_cast<uintptr_t>(dst[i]);
    if (bytes == 0) continue;
    r[n++] = {d, d + bytes, i, true};
    if (s != d) r[n++] = {s, s + bytes, i, false};
  }
  std::sort(r.get(), r.get() + n, [](const Range& a, const Range& b) { return a.from < b.from; });
  // the range before that ends last, of all and of the results
  const Range *any = nullptr, *result = nullptr;
  for (const Range* x = r.get(); x != r.get() + n; ++x) {
    const Range* y = x->result ? any : result;
    if (y && x->from < y->to)
      return fail(ISOLOCO_ERR_ALIAS, "tensors %d and %d: one's result overlaps the other", y->tensor, x->tensor);
    if (!any || x->to > any->to) any = x;
    if (x->result && (!result || x->to > result->to)) result = x;
  }
  return ISOLOCO_OK;
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

extern "C" {

isoloco_status isoloco_clip_workspace_size(int32_t n_tensors, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  if (n_tensors < 0) return fail(ISOLOCO_ERR_INVALID_ARG, "n_tensors = %d", n_tensors);
  *bytes = clip_workspace(n_tensors);
  return ISOLOCO_OK;
}

isoloco_status isoloco_clip_grads(const void* const* src, void* const* dst, const int64_t* counts,
                                  const int32_t* dtypes, int32_t n_tensors, float max_norm, float* norm,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (n_tensors < 0) return fail(ISOLOCO_ERR_INVALID_ARG, "n_tensors = %d", n_tensors);
  if (n_tensors && (!src || !counts || !dtypes)) return fail(ISOLOCO_ERR_INVALID_ARG, "NULL table");
  if (!norm) return fail(ISOLOCO_ERR_INVALID_ARG, "norm is NULL");
  if (!aligned_to(norm, 4)) return fail(ISOLOCO_ERR_ALIGN, "norm is not 4-byte aligned");
  if (!(max_norm >= 0.f)) return fail(ISOLOCO_ERR_INVALID_ARG, "max_norm = %g: zero or more is wanted", (double)max_norm);
  const size_t need = clip_workspace(n_tensors);
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  for (int i = 0; i < n_tensors; ++i) {
    if (counts[i] < 0 || counts[i] > (int64_t)1 << 40)
      return fail(ISOLOCO_ERR_INVALID_ARG, "tensor %d has %lld elements", i, (long long)counts[i]);
    if (!is_dtype(dtypes[i])) return fail(ISOLOCO_ERR_INVALID_ARG, "tensor %d: dtype %d", i, dtypes[i]);
    if (counts[i] == 0) continue;
    const size_t elem = dtype_bytes(dtypes[i]), bytes = (size_t)counts[i] * elem;
    if (!src[i] || (dst && !dst[i])) return fail(ISOLOCO_ERR_INVALID_ARG, "tensor %d is NULL", i);
    if (!aligned_to(src[i], elem) || (dst && !aligned_to(dst[i], elem)))
      return fail(ISOLOCO_ERR_ALIGN, "tensor %d is not aligned to its elements", i);
    if (dst && dst[i] != src[i] && ranges_overlap(src[i], bytes, dst[i], bytes))
      return fail(ISOLOCO_ERR_ALIAS, "tensor %d overlaps its result in part", i);
    if (ranges_overlap(src[i], bytes, workspace, need) || (dst && ranges_overlap(dst[i], bytes, workspace, need)))
      return fail(ISOLOCO_ERR_ALIAS, "tensor %d overlaps the workspace", i);
    if (ranges_overlap(src[i], bytes, norm, 8) || (dst && ranges_overlap(dst[i], bytes, norm, 8)))
      return fail(ISOLOCO_ERR_ALIAS, "tensor %d overlaps norm", i);
  }
  if (ranges_overlap(norm, 8, workspace, need)) return fail(ISOLOCO_ERR_ALIAS, "norm overlaps the workspace");
  if (dst && n_tensors > 1) ISOLOCO_TRY(check_results_apart(src, dst, counts, dtypes, n_tensors));
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double* part = static_cast<double*>(workspace);
  // Results apart from their sources go past the caches if both do not fit in them.  Both
  // sides measured, us of a call, and with a pass that scales the results after it, stored /
  // stored past: 32M float32 65 / 64 and 107 / 123, 110M bfloat16 116 / 100 and 300 / 285,
  // 888M bfloat16 1026 / 993 and 2345 / 2328.
  int64_t results = 0;
  for (int i = 0; dst && i < n_tensors; ++i)
    if (dst[i] != src[i]) results += counts[i] * (int64_t)dtype_bytes(dtypes[i]);
  int n_part = 0;
  for (int pass = 0; pass < (dst ? 2 : 1); ++pass) {
    bool first_launch = true;
    for (int at = 0; at < n_tensors;) {
      // the next tensors that hold something, as many as a launch takes (and whose chunks it can count)
      ClipArgs a;
      a.n = 0;
      a.in_place = 1;
      int64_t chunks = 0;
      for (; at < n_tensors && a.n < kClipTensors; ++at) {
        if (counts[at] == 0) continue;
        const int64_t bytes = counts[at] * (int64_t)dtype_bytes(dtypes[at]);
        const int64_t c = (bytes + kChunkBytes - 1) / kChunkBytes;
        if (chunks + c > INT32_MAX) break;
        a.src[a.n] = src[at];
        a.dst[a.n] = dst ? dst[at] : nullptr;
        a.in_place &= a.dst[a.n] == a.src[a.n];
        a.first[a.n] = (int32_t)chunks;
        a.last[a.n] = (int32_t)(bytes - (c - 1) * kChunkBytes);
        a.bf16[a.n] = dtypes[at] == ISOLOCO_BF16;
        chunks += c;
        ++a.n;
      }
      if (a.n == 0) break;
      a.first[a.n] = (int32_t)chunks;
      const int grid = (int)(chunks < kClipBlocks ? chunks : kClipBlocks);
      if (pass == 0) {
        hipLaunchKernelGGL(clip_norm_kernel, dim3(grid), dim3(kClipThreads), 0, st, a, part + n_part);
        n_part += grid;
      } else {
        hipLaunchKernelGGL(2 * results > kCacheBytes ? clip_scale_kernel<true> : clip_scale_kernel<false>, dim3(grid),
                           dim3(kClipThreads), 0, st, a, part, n_part, max_norm, first_launch ? norm : nullptr);
        first_launch = false;
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return hip_fail(e, "clipping");
    }
    // nothing was or will be scaled: the norm has a launch of its own
    if (pass == 0 && (!dst || n_part == 0)) {
      hipLaunchKernelGGL(clip_finish_kernel, dim3(1), dim3(256), 0, st, part, n_part, max_norm, norm);
      const hipError_t e = hipGetLastError();
      return e == hipSuccess ? ISOLOCO_OK : hip_fail(e, "clipping");
    }
  }
  return ISOLOCO_OK;
}

}  // extern "C"
