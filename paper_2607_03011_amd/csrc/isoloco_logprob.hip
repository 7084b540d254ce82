// Log probabilities of given tokens, with entropy and the best alternatives, and
// their gradient.  With x the logits of a row, m = max x, t_j = scale (x_j - m) log2 e:
//
//   s = sum_j 2^t_j,  w = sum_j 2^t_j t_j
//   lse = scale m + log s                   logprob = scale (x_target - m) - log s
//   entropy = log s - w log 2 / s
//   dlogits_j = scale (dlogprob (1[j = target] - p_j) - dentropy p_j (log p_j + entropy))
//
// Forward: one pass over a row with the running maximum and sums of its softmax.  The
// maximum is kept as a logit and taken from the logits before the scale: the largest
// one's t is then 0 whatever the products' rounding, which past |scale x| = 1e9 (masks
// that are written as a large number) is more than an exponential's range.
// A column of -infinity (a mask) has p = 0 and adds nothing; a row of nothing but
// those has lse = logprob = -infinity, entropy 0 and no gradient.  A NaN or a
// logit of +infinity makes the row's results NaN.
// Bounded by memory: the forward pass reads the logits once, the gradient reads
// them again and writes as much.
#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

constexpr float kLog2 = 0.69314718055994530942f;

// e^x, x <= 0 where it counts: the product's rounding moves the result by |x| ulps
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// 2^t is 0 from here on down: a product with it takes this for t (which may be -infinity)
constexpr float kNothing = -200.f;

// The softmax of some of a row's logits: their maximum m, and s and w as above against it
// ({-infinity, 0, 0} of nothing; a NaN or +infinity among them leaves a NaN in s).
// `rate` is rate_of(scale).
struct Soft {
  float m, s, w;
  __device__ __forceinline__ void raise(float to, float rate) {
    if (to == m) return;
    if (m != -INFINITY) {
      const float t = (m - to) * rate, e = __builtin_amdgcn_exp2f(t);
      w = e > 0.f ? e * (w + s * t) : 0.f;
      s = e * s;
    }
    m = to;
  }
  __device__ __forceinline__ void join(const Soft& o, float rate) {
    const float to = fmaxf(m, o.m);
    Soft b = o;
    raise(to, rate);
    b.raise(to, rate);
    s += b.s;
    w += b.w;
  }
};

constexpr int kMaxSplits = 64;

struct RowOut {
  float* logprob;
  float* entropy;
  float* lse;
  float* top_logprob;
  int64_t* top_index;
};

struct RowArgs {
  int64_t ld, vocab;
  float scale, rate;
  int top_k;
  int splits;      // workgroups per row
  int64_t span;    // a split's columns (a multiple of a vector's)
  Soft* part;      // splits > 1: each one's softmax, and its top_k keys
  uint64_t* keys;
  RowOut o;
};

constexpr int kHeld = 64;         // logits that a thread holds in registers
// (8 waves a SIMD in bfloat16 leave a workgroup of one 5 KiB of LDS)
constexpr int candidates_of(int waves) { return waves == 1 ? 512 : 1024; }

// A row's results, from its softmax and (top_k) its largest keys in falling order:
// thread i of the workgroup writes alternative i.
template <typename T, typename ID>
__device__ __forceinline__ void put_row(const RowArgs& g, const T* row, const ID* targets, int64_t r, const Soft& a) {
  const bool empty = a.m == -INFINITY && a.s == 0.f;
  const float log_s = logf(a.s);
  if (g.o.lse) g.o.lse[r] = empty ? -INFINITY : fmaf(a.m, g.scale, log_s);
  if (g.o.entropy) g.o.entropy[r] = empty ? 0.f : log_s - a.w * kLog2 / a.s;
  if (g.o.logprob) {
    const int64_t t = targets[r];
    float lp = 0.f;
    if (t >= 0 && t < g.vocab) lp = empty ? -INFINITY : ((float)row[t] - a.m) * g.scale - log_s;
    g.o.logprob[r] = lp;
  }
}
__device__ __forceinline__ void put_top(const RowArgs& g, int64_t r, int place, uint64_t key, const Soft& a) {
  const bool empty = a.m == -INFINITY && a.s == 0.f;
  g.o.top_logprob[r * g.top_k + place] = empty ? -INFINITY : (value_of(key) - a.m) * g.scale - logf(a.s);
  g.o.top_index[r * g.top_k + place] = index_of(key);
}

// One workgroup of WAVES waves per row, or per split of a row.
//
// Its columns are taken kHeld per thread at a time, as they are stored: the maximum of
// those, then their sums against it, 12 instructions' time per logit (4 of it the
// exponential) against the 14 that their bytes' time allows in bfloat16 (a running
// maximum per vector: 18).  Unpacked once, in twice the registers, it is 10, but 4 waves
// are on a SIMD instead of 8: 122 against 108 us for 8192 rows of 32000, 4.8 TB/s.
//
// Alternatives: the threads of one lane number are a group; the top_k-th largest of
// the 64 groups' maxima bounds the top_k-th largest logit from below, and few logits
// reach it.  Those are ranked by value and index.  Where more than kCandidates do
// (equal values, or all of the largest in few groups), the row is gone through once
// more per alternative.
template <typename T, typename ID, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, sizeof(T) == 2 ? 8 : 4)
    logprob_kernel(const T* logits, const ID* targets, RowArgs g) {
  constexpr int N = Vec<T>::N, kThreads = 64 * WAVES, kVecs = kHeld / N, kCandidates = candidates_of(WAVES);
  __shared__ Soft part[WAVES];
  __shared__ float group[WAVES][64];
  __shared__ uint64_t cand[kCandidates];
  __shared__ uint64_t wave_best[WAVES];
  __shared__ int n_cand;
  __shared__ int rank[64];
  const int64_t r = blockIdx.x / g.splits;
  const int split = (int)(blockIdx.x - r * g.splits);
  const int64_t begin = split * g.span;
  const int count = (int)min(g.span, g.vocab - begin), whole = count / N;  // (a row has at most 2^30)
  const T* row = logits + r * g.ld;
  const T* p = row + begin;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  // the threads' logits of one turn: vectors, then single ones at the end
  u32x4 v[kVecs];
  float last;
  const auto load = [&](int base) {
#pragma unroll
    for (int c = 0; c < kVecs; ++c) {
      const int i = base + c * kThreads + (int)threadIdx.x;
      v[c] = sizeof(T) == 2 ? (u32x4)(0xff80ff80u) : (u32x4)(0xff800000u);  // -infinity
      if (i < whole) v[c] = *reinterpret_cast<const u32x4_any*>(p + i * N);
    }
    const int at = whole * N + (int)threadIdx.x;
    last = base == 0 && at < count ? (float)p[at] : -INFINITY;
  };
  constexpr int turn = kThreads * kVecs;
  const bool once = whole <= turn;  // the registers hold all of it

  Soft a = {-INFINITY, 0.f, 0.f};
  for (int base = 0; base == 0 || base < whole; base += turn) {
    load(base);
    float most = last;
#pragma unroll
    for (int c = 0; c < kVecs; ++c)
      if (base + c * kThreads < whole) {
        float x[N];
        unpack<T>(v[c], x);
#pragma unroll
        for (int e = 0; e < N; ++e) most = fmaxf(most, x[e]);
      }
    // (unpacked again after this: as float32 they would take the registers of half the waves)
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int c = 0; c < kVecs; ++c) asm("" : "+v"(v[c]));
    }
    a.raise(fmaxf(a.m, most), g.rate);
    const float m = a.m == -INFINITY ? 0.f : a.m;
    const auto add = [&](float v) {
      const float t = (v - m) * g.rate, e = __builtin_amdgcn_exp2f(t);
      a.s += e;
      a.w = fmaf(e, fmaxf(t, kNothing), a.w);
    };
#pragma unroll
    for (int c = 0; c < kVecs; ++c)
      if (base + c * kThreads < whole) {
        float x[N];
        unpack<T>(v[c], x);
#pragma unroll
        for (int e = 0; e < N; ++e) add(x[e]);
      }
    if (base == 0) add(last);
  }
  Soft b = a;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    Soft o;
    o.m = __shfl_xor(b.m, off, 64);
    o.s = __shfl_xor(b.s, off, 64);
    o.w = __shfl_xor(b.w, off, 64);
    b.join(o, g.rate);
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) part[wave] = b;
  }
  if (g.top_k) {
    group[wave][lane] = a.m;
    if (wave == 0) rank[lane] = 0;
    if (threadIdx.x == 0) n_cand = 0;
  }
  __syncthreads();
  if constexpr (WAVES > 1) {
    b = part[0];
    for (int w = 1; w < WAVES; ++w) b.join(part[w], g.rate);
  }
  const bool whole_row = g.splits == 1;
  if (threadIdx.x == 0) {
    if (whole_row) put_row(g, row, targets, r, b);
    else g.part[blockIdx.x] = b;
  }
  if (!g.top_k) return;
  uint64_t* keys = g.keys + (int64_t)blockIdx.x * g.top_k;
  const auto put = [&](int place, uint64_t key) {
    if (whole_row) put_top(g, r, place, key, b);
    else keys[place] = key;
  };

  // (a NaN is above every maximum here: such rows go the long way)
  const bool odd = b.s != b.s;
  if (!odd) {
    // each wave ranks the groups among some of them (one wave alone: 114 against 108 us
    // for 4096 rows of 32000 in float32)
    float own = group[0][lane];
    for (int w = 1; w < WAVES; ++w) own = fmaxf(own, group[w][lane]);
    int above = 0;
#pragma unroll
    for (int q = 0; q < 64 / WAVES; ++q) {
      const int i = wave * (64 / WAVES) + q;
      const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own), i));
      above += other > own || (other == own && i < lane);
    }
    if constexpr (WAVES > 1) {
      atomicAdd(&rank[lane], above);
      __syncthreads();
      above = rank[lane];
    }
    const uint64_t at_bound = __ballot(above == g.top_k - 1);
    const float bound = __uint_as_float(
        __builtin_amdgcn_readlane(__float_as_uint(own), __ffsll((unsigned long long)at_bound) - 1));
    const auto take = [&](float v, int i) {
      if (v >= bound) {
        const int c = atomicAdd(&n_cand, 1);
        if (c < kCandidates) cand[c] = key_of(v, (uint32_t)(begin + i));
      }
    };
    for (int base = 0; base == 0 || base < whole; base += turn) {
      if (!once) load(base);
#pragma unroll
      for (int c = 0; c < kVecs; ++c) {
        const int i = base + c * kThreads + (int)threadIdx.x;
        float x[N];
        unpack<T>(v[c], x);
        float most = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, x[e]);
        if (most >= bound && i < whole) {
#pragma unroll
          for (int e = 0; e < N; ++e) take(x[e], i * N + e);
        }
      }
      const int at = whole * N + (int)threadIdx.x;
      if (base == 0 && at < count) take(last, at);
    }
  }
  __syncthreads();
  const int n = n_cand;
  // (a split may hold fewer columns than alternatives are wanted: the keys after them are 0)
  const int have = min(g.top_k, count);
  if (threadIdx.x >= have && threadIdx.x < g.top_k) keys[threadIdx.x] = 0;
  if (!odd && n <= kCandidates) {
    for (int c = threadIdx.x; c < n; c += kThreads) {
      const uint64_t k = cand[c];
      int above = 0;
      for (int i = 0; i < n; ++i) above += cand[i] > k;
      if (above < have) put(above, k);
    }
    return;
  }
  uint64_t below = 0;
  for (int j = 0; j < have; ++j) {
    uint64_t most = 0;
    for (int i = threadIdx.x; i < count; i += kThreads) {
      const uint64_t k = key_of((float)p[i], (uint32_t)(begin + i));
      if (j == 0 || k < below) most = max64(most, k);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = max64(most, (uint64_t)__shfl_xor((unsigned long long)most, off, 64));
    __syncthreads();
    if (lane == 0) wave_best[wave] = most;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) most = max64(most, wave_best[w]);
    if (threadIdx.x == 0) put(j, most);
    below = most;
  }
}

// A row's splits joined, in their order.
template <typename T, typename ID>
__global__ void __launch_bounds__(256) logprob_join_kernel(const T* logits, const ID* targets, RowArgs g) {
  __shared__ uint64_t keys[kMaxSplits * ISOLOCO_MAX_TOP];
  const int64_t r = blockIdx.x;
  const Soft* part = g.part + r * g.splits;
  Soft a = part[0];
  for (int i = 1; i < g.splits; ++i) a.join(part[i], g.rate);
  if (threadIdx.x == 0) put_row(g, logits + r * g.ld, targets, r, a);
  const int n = g.splits * g.top_k;
  for (int i = threadIdx.x; i < n; i += 256) keys[i] = g.keys[r * n + i];
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const uint64_t k = keys[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += keys[j] > k;
    if (k && above < g.top_k) put_top(g, r, above, k, a);
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

// p is formed from the lse, a float32: off by 2^-24 |lse| of itself, and for masks written
// as a large number all of it.  From here on a row's maximum and sum are formed again: in
// float32 where p would be off by 2^-16, in bfloat16 by 2^-11, a quarter of the result's
// rounding.  (Us for rows of 32000 above and below the line: 8192 in bfloat16 628 and 181,
// 4096 in float32 610 and 185, for three readings instead of one.)
template <typename T>
constexpr float kSureLse = sizeof(T) == 2 ? 8192.f : 256.f;

// The row's gradient without its lse: its maximum and sum against that, then the gradient,
// by one workgroup (in place, nobody else may read the row).  grad(log p, column).  An lse
// that the row's own sum cannot have been rounded to is of more than this row (a vocabulary
// in parts): it is taken as it is.
template <typename T, typename Grad>
__device__ __forceinline__ void grad_of_row(const T* row, T* out, int64_t vocab, float scale, float lse,
                                            const Grad& grad) {
  constexpr int N = Vec<T>::N, kWaves = kGradThreads / 64, kAtOnce = 4;
  __shared__ float most_of[kWaves], sum_of[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t whole = vocab / N, rest = whole * N + threadIdx.x;
  // take(logits, first column) of the thread's vectors
  const auto vectors = [&](const auto& take) {
    for (int64_t base = threadIdx.x; base < whole; base += kAtOnce * kGradThreads) {
      u32x4 v[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t i = base + u * kGradThreads;
        if (i < whole) v[u] = *reinterpret_cast<const u32x4_any*>(row + i * N);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t i = base + u * kGradThreads;
        float x[N];
        unpack<T>(v[u], x);
        if (i < whole) take(x, i * N);
      }
    }
  };
  float m = rest < vocab ? (float)row[rest] : -INFINITY, s = 0.f;
  vectors([&](const float* x, int64_t) {
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, x[e]);
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if (lane == 0) most_of[wave] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, most_of[w]);
  const bool empty = m == -INFINITY;
  if (!empty) {
    const float rate = rate_of(scale);
    const auto term = [&](float x) { return __builtin_amdgcn_exp2f((x - m) * rate); };
    if (rest < vocab) s = term((float)row[rest]);
    vectors([&](const float* x, int64_t) {
#pragma unroll
      for (int e = 0; e < N; ++e) s += term(x[e]);
    });
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if (lane == 0) sum_of[wave] = s;
  __syncthreads();
  s = 0.f;
  for (int w = 0; w < kWaves; ++w) s += sum_of[w];
  const float own = logf(s), given = fmaf(-m, scale, lse);
  const float log_s = isinf(lse) || fabsf(given - own) <= fmaf(fabsf(lse), 0x1p-23f, 0x1p-16f) ? own : given;
  const auto grad_of = [&](float x, int64_t i) { return empty ? 0.f : grad((x - m) * scale - log_s, i); };
  vectors([&](const float* x, int64_t i) {
    float d[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = grad_of(x[e], i + e);
    *reinterpret_cast<u32x4_any*>(out + i) = pack<T>(d);
  });
  if (rest < vocab) out[rest] = (T)grad_of((float)row[rest], rest);
}

// One workgroup per row and span of kGradThreads * kGradVecs vectors.  PAST: the result
// goes past the caches.
template <typename T, typename ID, bool PAST>
__global__ void __launch_bounds__(kGradThreads) logprob_grad_kernel(const T* logits, int64_t ld, int64_t rows, int64_t vocab,
                                                                    const ID* targets, float scale, GradIn in,
                                                                    T* dlogits, int64_t ld_d, int spans) {
  constexpr int N = Vec<T>::N;
  // (the last rows first: the forward pass read them last, some are still in a cache)
  const int64_t r = rows - 1 - blockIdx.x / spans, first = (int64_t)(blockIdx.x % spans) * (kGradThreads * kGradVecs);
  const T* row = logits + r * ld;
  T* out = dlogits + r * ld_d;
  const float lse = in.lse[r];
  const int64_t t = targets ? (int64_t)targets[r] : -1;
  const bool given = t >= 0 && t < vocab;
  const float dl = given ? in.dlogprob[r] : 0.f;
  const float de = in.dentropy ? in.dentropy[r] : 0.f, h = in.dentropy ? in.entropy[r] : 0.f;
  // nothing to hand back: the row's logits are not read
  const bool none = dl == 0.f && de == 0.f;
  const auto grad_at = [&](float lp, int64_t i) {
    const float p = exp_of(lp);
    float d = (i == t ? 1.f : 0.f) - p;
    d *= dl;
    if (p > 0.f) d -= de * (p * (lp + h));
    return d * scale;
  };
  if (!none && fabsf(lse) >= kSureLse<T>) {
    // one of the row's workgroups, another one from row to row: their XCDs take turns
    if ((int)(blockIdx.x % spans) == (int)(r % spans)) grad_of_row(row, out, vocab, scale, lse, grad_at);
    return;
  }
  const auto grad = [&](float x, int64_t i) { return grad_at(fmaf(x, scale, -lse), i); };
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
      v = pack<T>(x);
      u32x4_any* to = reinterpret_cast<u32x4_any*>(out + i * N);
      if constexpr (PAST) __builtin_nontemporal_store(v, to);
      else *to = v;
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

// Workgroups per row: one, unless the rows are few and long.  Both sides measured, us a
// call of a graph with 8 alternatives in bfloat16, 1 / 2 / 4 / 8 splits:
//           1 row                      64 rows                    127 or 256 rows
//    32000  8.5 / 9.6 / 9.7 / 12.3     9.3 / 10.9 / 10.8 / 13.5   11.0 / 14.4 / 15.4 / 17.5 (256)
//    50257  11.4 / 10.4 / 10.1 / 10.7  14.2 / 12.4 / 11.9 / 12.9  14.6 / 13.2 / 14.2 / 16.1 (127),
//                                                                 15.7 / 16.7 / 17.8 / 21.4 (256)
//   128000  19.3 / 14.6 / 11.4 / 11.4  20.9 / 17.0 / 14.6 / 15.8  22.3 / 18.8 / 18.3 / 19.5 (127),
//                                                                 27.0 / 27.7 / 25.3 / 26.5 (256)
// (Without a graph the second launch costs the host 4 us more: one row of 50257 12.5 whole,
// 17.0 in splits.)
int splits_of(int64_t rows, int64_t vocab) {
  if (rows >= 128 || vocab <= 40000) return 1;
  const int64_t most = vocab / 8192, wanted = 512 / (rows ? rows : 1);
  const int64_t s = most < wanted ? most : wanted;
  return (int)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s);
}

size_t logprob_workspace(int64_t rows, int64_t vocab, int top_k) {
  const size_t s = (size_t)splits_of(rows, vocab);
  return s > 1 ? (size_t)rows * s * (16 + 8 * (size_t)top_k) : 0;
}

// the fewest that hold a row (or split) at once, if any do
int threads_of(int64_t span) { return span <= 64 * kHeld ? 64 : span <= 256 * kHeld ? 256 : 512; }

template <typename T, typename ID>
void run_forward(const void* logits, const void* targets, int64_t rows, const RowArgs& g, hipStream_t st) {
  const T* l = static_cast<const T*>(logits);
  const ID* t = static_cast<const ID*>(targets);
  const dim3 grid((unsigned)(rows * g.splits));
  const int threads = threads_of(g.span);
  if (threads == 64) hipLaunchKernelGGL((logprob_kernel<T, ID, 1>), grid, dim3(64), 0, st, l, t, g);
  else if (threads == 256) hipLaunchKernelGGL((logprob_kernel<T, ID, 4>), grid, dim3(256), 0, st, l, t, g);
  else hipLaunchKernelGGL((logprob_kernel<T, ID, 8>), grid, dim3(512), 0, st, l, t, g);
  if (g.splits > 1) hipLaunchKernelGGL((logprob_join_kernel<T, ID>), dim3((unsigned)rows), dim3(256), 0, st, l, t, g);
}

template <typename T, typename ID>
void run_grad(const void* logits, int64_t ld, int64_t rows, int64_t vocab, const void* targets, float scale,
              const GradIn& in, void* dlogits, int64_t ld_d, int spans, hipStream_t st) {
  // Both sides measured, stored past the caches / stored, us of both passes over rows of 32000
  // in bfloat16, and with a pass that scales the gradient after them: 8192 rows 273 / 301 and
  // 469 / 477; 4096 rows (just below the line) 129 / 153 and 236 / 241; 2048 rows 73 / 74 and
  // 113 / 109.
  const bool past = dlogits != logits && rows * vocab * (int64_t)sizeof(T) > kCacheBytes;
  hipLaunchKernelGGL((past ? logprob_grad_kernel<T, ID, true> : logprob_grad_kernel<T, ID, false>), dim3((unsigned)(rows * spans)), dim3(kGradThreads), 0, st,
                     static_cast<const T*>(logits), ld, rows, vocab, static_cast<const ID*>(targets), scale, in,
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
  *bytes = logprob_workspace(rows, vocab, top_k);
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
  const size_t need = logprob_workspace(rows, vocab, top_k);
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  if (ranges_overlap(workspace, need, logits, nb) ||
      ranges_overlap(workspace, need, targets, targets ? (size_t)rows * index_bytes(target_type) : 0))
    return fail(ISOLOCO_ERR_ALIAS, "the workspace overlaps an input");
  for (const auto& x : outs)
    if (ranges_overlap(workspace, need, x.p, x.bytes)) return fail(ISOLOCO_ERR_ALIAS, "the workspace overlaps %s", x.name);
  RowArgs g;
  g.ld = ld_logits;
  g.vocab = vocab;
  g.scale = scale;
  g.rate = rate_of(scale);
  g.top_k = top_k;
  g.splits = splits_of(rows, vocab);
  g.span = ((vocab + g.splits - 1) / g.splits + 7) / 8 * 8;
  g.splits = (int)((vocab + g.span - 1) / g.span);
  g.keys = static_cast<uint64_t*>(workspace);
  g.part = reinterpret_cast<Soft*>(g.keys + rows * g.splits * top_k);
  g.o = {logprob, entropy, lse, top_logprob, top_index};
  if (!launchable(rows * g.splits, threads_of(g.span))) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many rows for one launch");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_forward, logits, targets, rows, g, st);
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
  if (!launchable(rows * spans, kGradThreads)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  const GradIn in = {lse, entropy, dlogprob, dentropy};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_grad, logits, ld_logits, rows, vocab, targets, scale, in, dlogits, ld_dlogits, (int)spans, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "gradient of token log probabilities");
}

}  // extern "C"
