// Log probabilities of given tokens, with entropy and the best alternatives, and
// their gradient.  With z = scale * logits of a row, m = max z:
//
//   lse = m + log sum_j e^(z_j - m)         logprob = z_target - lse
//   entropy = log s - w / s,  s = sum e^(z_j - m),  w = sum e^(z_j - m) (z_j - m)
//   dlogits_j = scale (dlogprob (1[j = target] - p_j) - dentropy p_j (log p_j + entropy))
//
// Forward: one pass over a row with the running maximum and sums of its softmax.
// A column of -infinity (a mask) has p = 0 and adds nothing; a row of nothing but
// those has lse = logprob = -infinity, entropy 0 and no gradient.  A NaN or a
// logit of +infinity makes the row's results NaN.
// Bounded by memory: the forward pass reads the logits once, the gradient reads
// them again and writes as much.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "isoloco_device.h"
#include "isoloco_error.h"

namespace isoloco {
namespace {

typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr float kLog2e = 1.44269504088896340736f;

// e^x, x <= 0 where it counts: the product's rounding moves the result by |x| ulps
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// The running softmax of one thread: m is the largest z so far, s and w as above
// ({-infinity, 0, 0} before the first).
struct Soft {
  float m, s, w;
  // both sums on the new maximum (both -infinity: nothing was summed; a NaN or
  // +infinity gets through the exponential and stays)
  __device__ __forceinline__ void raise(float to) {
    if (to == m) return;
    if (m != -INFINITY) {
      const float d = m - to, e = exp_of(d);
      w = e > 0.f ? e * (w + s * d) : 0.f;  // (s d may leave the range where e is 0)
      s = e * s;
    }
    m = to;
  }
  __device__ __forceinline__ void add(float z) {
    if (z == -INFINITY) return;
    const float d = z - m, e = exp_of(d);
    s += e;
    if (e > 0.f) w += e * d;
  }
  __device__ __forceinline__ void join(const Soft& o) {
    const float to = fmaxf(m, o.m);
    Soft b = o;
    raise(to);
    b.raise(to);
    s += b.s;
    w += b.w;
  }
};

// The order of the values: of equal ones (-0 and 0 among them) the lower index is
// the larger key; NaN is above all.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) {
  uint32_t u = __float_as_uint(x + 0.f);
  u = x != x ? 0xffffffffu : ((u >> 31) ? ~u : (u | 0x80000000u));
  return ((uint64_t)u << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int off) {
  return (uint64_t)__shfl_xor((unsigned long long)v, off, 64);
}

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kCandidates = 1024;

template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
};
template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[Vec<T>::N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = bf16_to_f32(v[i] & 0xffffu);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(v[i]);
    }
  }
}

// Calls f(logit, index) for the row's elements that a thread reads: 16-byte vectors
// in turn, then single elements at the end.
template <typename T, typename F>
__device__ __forceinline__ void each_logit(const T* row, int64_t vocab, F f) {
  constexpr int N = Vec<T>::N;
  const int64_t whole = vocab / N;
  for (int64_t i = threadIdx.x; i < whole; i += kRowThreads) {
    float x[N];
    unpack<T>(*reinterpret_cast<const u32x4_any*>(row + i * N), x);
#pragma unroll
    for (int e = 0; e < N; ++e) f(x[e], (uint32_t)(i * N + e));
  }
  const int64_t at = whole * N + threadIdx.x;
  if (at < vocab) f((float)row[at], (uint32_t)at);
}

struct RowOut {
  float* logprob;
  float* entropy;
  float* lse;
  float* top_logprob;
  int64_t* top_index;
};

// One workgroup per row.
template <typename T, typename ID>
__global__ void __launch_bounds__(kRowThreads) logprob_kernel(const T* logits, int64_t ld, int64_t vocab,
                                                              const ID* targets, float scale, int top_k, RowOut o) {
  __shared__ Soft part[kRowWaves];
  __shared__ uint64_t best[kRowWaves][64];
  __shared__ uint64_t cand[kCandidates];
  __shared__ uint64_t wave_best[kRowWaves];
  __shared__ int n_cand;
  const int64_t r = blockIdx.x;
  const T* row = logits + r * ld;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  Soft a = {-INFINITY, 0.f, 0.f};
  uint64_t own = 0;
  {
    constexpr int N = Vec<T>::N;
    const int64_t whole = vocab / N;
    for (int64_t i = threadIdx.x; i < whole; i += kRowThreads) {
      float x[N];
      unpack<T>(*reinterpret_cast<const u32x4_any*>(row + i * N), x);
      float to = a.m;
#pragma unroll
      for (int e = 0; e < N; ++e) to = fmaxf(to, x[e] * scale);
      a.raise(to);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        a.add(x[e] * scale);
        if (top_k) own = max64(own, key_of(x[e], (uint32_t)(i * N + e)));
      }
    }
    const int64_t at = whole * N + threadIdx.x;
    if (at < vocab) {
      const float x = (float)row[at];
      a.raise(fmaxf(a.m, x * scale));
      a.add(x * scale);
      if (top_k) own = max64(own, key_of(x, (uint32_t)at));
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    Soft b;
    b.m = __shfl_xor(a.m, off, 64);
    b.s = __shfl_xor(a.s, off, 64);
    b.w = __shfl_xor(a.w, off, 64);
    a.join(b);
  }
  if (lane == 0) part[wave] = a;
  if (top_k) {
    best[wave][lane] = own;
    if (threadIdx.x == 0) n_cand = 0;
  }
  __syncthreads();
  a = part[0];
  for (int w = 1; w < kRowWaves; ++w) a.join(part[w]);
  const bool empty = a.m == -INFINITY && a.s == 0.f;  // (a NaN is in s)
  const float log_s = logf(a.s), lse = empty ? -INFINITY : a.m + log_s;
  if (threadIdx.x == 0) {
    if (o.lse) o.lse[r] = lse;
    if (o.entropy) o.entropy[r] = empty ? 0.f : log_s - a.w / a.s;
    if (o.logprob) {
      const int64_t t = targets[r];
      float lp = 0.f;
      if (t >= 0 && t < vocab) lp = empty ? -INFINITY : (float)row[t] * scale - a.m - log_s;
      o.logprob[r] = lp;
    }
  }
  if (!top_k) return;

  // The threads of one lane number are a group; the top_k-th largest of the 64
  // groups' largest keys bounds the top_k-th largest of all from below, and few
  // keys are at or above it.
  for (int w = 0; w < kRowWaves; ++w) own = max64(own, best[w][lane]);
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < 64; ++i) {
    const uint64_t other = (uint64_t)__shfl((unsigned long long)own, i, 64);
    rank += other > own || (other == own && i < lane);
  }
  const uint64_t at = __ballot(rank == top_k - 1);
  const uint64_t bound = (uint64_t)__shfl((unsigned long long)own, __ffsll((unsigned long long)at) - 1, 64);
  each_logit(row, vocab, [&](float x, uint32_t i) {
    const uint64_t k = key_of(x, i);
    if (k >= bound) {
      const int c = atomicAdd(&n_cand, 1);
      if (c < kCandidates) cand[c] = k;
    }
  });
  __syncthreads();
  const int n = n_cand;
  if (n <= kCandidates) {
    for (int c = threadIdx.x; c < n; c += kRowThreads) {
      const uint64_t k = cand[c];
      int above = 0;
      for (int i = 0; i < n; ++i) above += cand[i] > k;
      if (above < top_k) {
        o.top_logprob[r * top_k + above] = empty ? -INFINITY : value_of(k) * scale - a.m - log_s;
        o.top_index[r * top_k + above] = (int64_t)(uint32_t)~(uint32_t)k;
      }
    }
    return;
  }
  // The largest values stand in few of the groups: one pass over the row per alternative.
  uint64_t below = ~0ull;
  for (int j = 0; j < top_k; ++j) {
    uint64_t most = 0;
    each_logit(row, vocab, [&](float x, uint32_t i) {
      const uint64_t k = key_of(x, i);
      if (k < below) most = max64(most, k);
    });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = max64(most, shfl_xor64(most, off));
    __syncthreads();
    if (lane == 0) wave_best[wave] = most;
    __syncthreads();
    for (int w = 0; w < kRowWaves; ++w) most = max64(most, wave_best[w]);
    if (threadIdx.x == 0) {
      o.top_logprob[r * top_k + j] = empty ? -INFINITY : value_of(most) * scale - a.m - log_s;
      o.top_index[r * top_k + j] = (int64_t)(uint32_t)~(uint32_t)most;
    }
    below = most;
  }
}

struct GradIn {
  const float* lse;
  const float* entropy;
  const float* dlogprob;
  const float* dentropy;
};

constexpr int kGradThreads = 256;
constexpr int kGradVecs = 4;  // 16-byte vectors of a thread

// One workgroup per row and span of kGradThreads * kGradVecs vectors.
template <typename T, typename ID>
__global__ void __launch_bounds__(kGradThreads) logprob_grad_kernel(const T* logits, int64_t ld, int64_t vocab,
                                                                    const ID* targets, float scale, GradIn in,
                                                                    T* dlogits, int64_t ld_d, int spans) {
  constexpr int N = Vec<T>::N;
  const int64_t r = blockIdx.x / spans, first = (int64_t)(blockIdx.x % spans) * (kGradThreads * kGradVecs);
  const T* row = logits + r * ld;
  T* out = dlogits + r * ld_d;
  const float lse = in.lse[r];
  const int64_t t = targets ? (int64_t)targets[r] : -1;
  const bool given = t >= 0 && t < vocab;
  const float dl = given ? in.dlogprob[r] : 0.f;
  const float de = in.dentropy ? in.dentropy[r] : 0.f, h = in.dentropy ? in.entropy[r] : 0.f;
  // nothing to hand back: the row's logits are not read
  const bool none = lse == -INFINITY || (dl == 0.f && de == 0.f);
  const auto grad = [&](float x, int64_t i) {
    const float lp = x * scale - lse, p = exp_of(lp);
    float d = (i == t ? 1.f : 0.f) - p;
    d *= dl;
    if (p > 0.f) d -= de * (p * (lp + h));
    return d * scale;
  };
  const int64_t whole = vocab / N;
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int64_t i = first + u * kGradThreads + threadIdx.x;
    if (i < whole) {
      u32x4 v = {};
      float x[N];
      if (!none) v = *reinterpret_cast<const u32x4_any*>(row + i * N);
      unpack<T>(v, x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = none ? 0.f : grad(x[e], i * N + e);
      if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){x[2 * e], x[2 * e + 1]}, bf16x2_t));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
      }
      *reinterpret_cast<u32x4_any*>(out + i * N) = v;
    }
  }
  const int64_t at = whole * N + threadIdx.x;
  if (first == 0 && at < vocab) out[at] = (T)(none ? 0.f : grad((float)row[at], at));
}

isoloco_status check_rows(int64_t rows, int64_t vocab, int32_t dtype, int32_t target_type, float scale) {
  if (rows < 0 || rows > kMaxExtent / 2 || vocab < 1 || vocab > kMaxExtent / 2)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of %lld logits", (long long)rows, (long long)vocab);
  if (!is_dtype(dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", dtype);
  if (!is_index_type(target_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "target type %d", target_type);
  if (!(scale > 0.f) || isinf(scale)) return fail(ISOLOCO_ERR_INVALID_ARG, "scale = %g: a positive number is wanted", (double)scale);
  return ISOLOCO_OK;
}

template <typename T, typename ID>
void run_forward(const void* logits, int64_t ld, int64_t rows, int64_t vocab, const void* targets, float scale,
                 int top_k, const RowOut& o, hipStream_t st) {
  hipLaunchKernelGGL((logprob_kernel<T, ID>), dim3((unsigned)rows), dim3(kRowThreads), 0, st,
                     static_cast<const T*>(logits), ld, vocab, static_cast<const ID*>(targets), scale, top_k, o);
}

template <typename T, typename ID>
void run_grad(const void* logits, int64_t ld, int64_t rows, int64_t vocab, const void* targets, float scale,
              const GradIn& in, void* dlogits, int64_t ld_d, int spans, hipStream_t st) {
  hipLaunchKernelGGL((logprob_grad_kernel<T, ID>), dim3((unsigned)(rows * spans)), dim3(kGradThreads), 0, st,
                     static_cast<const T*>(logits), ld, vocab, static_cast<const ID*>(targets), scale, in,
                     static_cast<T*>(dlogits), ld_d, spans);
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

#define BY_TYPES(RUN, ...)                                                             \
  do {                                                                                 \
    if (dtype == ISOLOCO_F32) {                                                        \
      if (target_type == ISOLOCO_I32) RUN<float, int32_t>(__VA_ARGS__);                \
      else RUN<float, int64_t>(__VA_ARGS__);                                           \
    } else {                                                                           \
      if (target_type == ISOLOCO_I32) RUN<__bf16, int32_t>(__VA_ARGS__);               \
      else RUN<__bf16, int64_t>(__VA_ARGS__);                                          \
    }                                                                                  \
  } while (0)

extern "C" {

isoloco_status isoloco_token_logprobs_workspace_size(int64_t rows, int64_t vocab, int32_t top_k, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  ISOLOCO_TRY(check_rows(rows, vocab, ISOLOCO_F32, ISOLOCO_I32, 1.f));
  if (top_k < 0 || top_k > ISOLOCO_MAX_TOP || top_k > vocab) return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d", top_k);
  *bytes = 0;
  return ISOLOCO_OK;
}

isoloco_status isoloco_token_logprobs(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                      int64_t vocab, const void* targets, int32_t target_type, float scale,
                                      int32_t top_k, float* logprob, float* entropy, float* lse, float* top_logprob,
                                      int64_t* top_index, void* workspace, size_t workspace_bytes,
                                      void* hip_stream) {
  ISOLOCO_TRY(check_rows(rows, vocab, dtype, target_type, scale));
  if (top_k < 0 || top_k > ISOLOCO_MAX_TOP || top_k > vocab)
    return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d of %lld, at most %d", top_k, (long long)vocab, ISOLOCO_MAX_TOP);
  if ((logprob != nullptr) != (targets != nullptr) && rows)
    return fail(ISOLOCO_ERR_INVALID_ARG, "targets and logprob go together");
  if (top_k && rows && (!top_logprob || !top_index))
    return fail(ISOLOCO_ERR_INVALID_ARG, "top_logprob or top_index is NULL");
  if (rows == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype);
  ISOLOCO_TRY(check_matrix("logits", logits, rows, vocab, ld_logits, e));
  if (targets) ISOLOCO_TRY(check_matrix("targets", targets, rows, 1, 1, index_bytes(target_type)));
  const size_t nb = matrix_bytes(rows, vocab, ld_logits, e), r4 = (size_t)rows * 4;
  const struct { const void* p; size_t bytes, align; const char* name; } outs[] = {
      {logprob, logprob ? r4 : 0, 4, "logprob"}, {entropy, entropy ? r4 : 0, 4, "entropy"}, {lse, lse ? r4 : 0, 4, "lse"},
      {top_logprob, r4 * top_k, 4, "top_logprob"}, {top_index, 2 * r4 * top_k, 8, "top_index"}};
  for (const auto& x : outs) {
    if (x.bytes && !aligned_to(x.p, x.align)) return fail(ISOLOCO_ERR_ALIGN, "%s is not aligned to its elements", x.name);
    if (ranges_overlap(x.p, x.bytes, logits, nb) ||
        ranges_overlap(x.p, x.bytes, targets, targets ? (size_t)rows * index_bytes(target_type) : 0))
      return fail(ISOLOCO_ERR_ALIAS, "%s overlaps an input", x.name);
    for (const auto* y = outs; y != &x; ++y)
      if (ranges_overlap(x.p, x.bytes, y->p, y->bytes)) return fail(ISOLOCO_ERR_ALIAS, "%s overlaps %s", x.name, y->name);
  }
  (void)workspace;
  (void)workspace_bytes;
  const RowOut o = {logprob, entropy, lse, top_logprob, top_index};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_forward, logits, ld_logits, rows, vocab, targets, scale, top_k, o, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "token log probabilities");
}

isoloco_status isoloco_token_logprobs_backward(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                               int64_t vocab, const void* targets, int32_t target_type, float scale,
                                               const float* lse, const float* entropy, const float* dlogprob,
                                               const float* dentropy, void* dlogits, int64_t ld_dlogits,
                                               void* hip_stream) {
  ISOLOCO_TRY(check_rows(rows, vocab, dtype, target_type, scale));
  if (rows == 0) return ISOLOCO_OK;
  if (!lse) return fail(ISOLOCO_ERR_INVALID_ARG, "lse is NULL");
  if ((targets != nullptr) != (dlogprob != nullptr)) return fail(ISOLOCO_ERR_INVALID_ARG, "targets and dlogprob go together");
  if (dentropy && !entropy) return fail(ISOLOCO_ERR_INVALID_ARG, "dentropy needs entropy");
  const size_t e = dtype_bytes(dtype);
  ISOLOCO_TRY(check_matrix("logits", logits, rows, vocab, ld_logits, e));
  ISOLOCO_TRY(check_matrix("dlogits", dlogits, rows, vocab, ld_dlogits, e));
  if (targets) ISOLOCO_TRY(check_matrix("targets", targets, rows, 1, 1, index_bytes(target_type)));
  const size_t nb = matrix_bytes(rows, vocab, ld_logits, e), db = matrix_bytes(rows, vocab, ld_dlogits, e);
  // in place: every element is read before it is written
  if (!(dlogits == logits && ld_dlogits == ld_logits) && ranges_overlap(dlogits, db, logits, nb))
    return fail(ISOLOCO_ERR_ALIAS, "dlogits overlaps the logits in part");
  const struct { const void* p; size_t bytes, align; const char* name; } ins[] = {
      {targets, targets ? (size_t)rows * index_bytes(target_type) : 0, index_bytes(target_type), "targets"},
      {lse, (size_t)rows * 4, 4, "lse"}, {entropy, dentropy ? (size_t)rows * 4 : 0, 4, "entropy"},
      {dlogprob, dlogprob ? (size_t)rows * 4 : 0, 4, "dlogprob"}, {dentropy, dentropy ? (size_t)rows * 4 : 0, 4, "dentropy"}};
  for (const auto& x : ins) {
    if (x.bytes && !aligned_to(x.p, x.align)) return fail(ISOLOCO_ERR_ALIGN, "%s is not aligned to its elements", x.name);
    if (ranges_overlap(dlogits, db, x.p, x.bytes)) return fail(ISOLOCO_ERR_ALIAS, "dlogits overlaps %s", x.name);
  }
  const int64_t vecs = vocab / (16 / (int64_t)e);
  const int64_t spans = vecs == 0 ? 1 : (vecs + kGradThreads * kGradVecs - 1) / (kGradThreads * kGradVecs);
  if (rows * spans > INT32_MAX) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  const GradIn in = {lse, entropy, dlogprob, dentropy};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_grad, logits, ld_logits, rows, vocab, targets, scale, in, dlogits, ld_dlogits, (int)spans, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "gradient of token log probabilities");
}

}  // extern "C"
