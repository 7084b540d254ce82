// Distillation from a teacher's most likely tokens: the loss of each row and its
// gradient in the student's logits.  With x the logits of a row, z = scale x, q their
// softmax, and t_i the teacher's log probabilities of the columns c_i:
//
//   drop     p_i = e^t_i / sum_i e^t_i                loss = sum_i p_i (log p_i - log q_ci)
//   bucket   p_i = e^t_i, p_r = 1 - sum_i p_i         loss = the same + p_r (log p_r - log q_r)
//            with q_r the sum of q over the columns that are not listed
//
//   W = sum_i p_i (+ p_r);  dz_j = q_j W - sum of the p_i with c_i = j, less p_r q_j / q_r
//   where j is not listed
//
// With M the maximum over the columns that are not listed, A the sum of their e^((x_j - M) scale)
// and S that of all against the row's maximum m, those columns' gradient is
//
//   dz_j = c e^((x_j - M) scale),   c = W e^((M - m) scale) / S - p_r / A
//
// one exponential against their own maximum: against the row's it is 0 in float32 once they lie
// 87 / scale below it, where p_r / q_r is past float32 and the product is still their share of p_r.
//
// The loss is the difference of nearly equal numbers once the student has learnt, so what
// is formed once a row is formed in 64 bits; the sums over the vocabulary are of float32
// exponentials.  q_r is summed from the columns that are not listed, not taken as one less
// the others (which leaves nothing of a small one): the listed columns are marked in a
// bitmap in LDS, and the pass over the row takes a marked column for -infinity.
//
// float32 logits take that path without q_r too: the listed columns, which are most of the sum
// once the student agrees, are then summed in 64 bits.
//
// Bounded by memory: the loss reads the logits once, the gradient reads them again and
// writes as much.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

constexpr int kMaxSplits = 64;
constexpr int kHeld = 64;               // logits that a thread holds in registers
constexpr int64_t kMostSpan = 1 << 17;  // columns of a workgroup with a bitmap: 16 KiB of it
constexpr int kHalfTurns = 2;          // of 256 threads, see threads_of
constexpr int kPerLane = (ISOLOCO_MAX_TEACHER + 63) / 64;

// scale log2 e in two floats, and the distance from which on its power of 2 is 0.
struct Rate {
  float hi, lo, least;
};
Rate rate_parts(float scale) {
  const float hi = rate_of(scale);
  const double lo = (double)scale * 1.4426950408889634074 - hi;
  // (finite: a masked logit is at -infinity, however small the scale)
  return {hi, hi == FLT_MAX ? 0.f : (float)lo, fmaxf(-200.f / hi, -FLT_MAX)};
}

// e^(d scale), d <= 0.  EXACT: to float32's last bits, for float32 logits (the rounding of the
// product alone moves the plain one by |d scale| of them); bfloat16 ones do not need it.
template <bool EXACT>
__device__ __forceinline__ float power(float d, const Rate& r) {
  if constexpr (!EXACT) return __builtin_amdgcn_exp2f(d * r.hi);
  const float n = __builtin_rintf(d * r.hi), e = ldexpf(__builtin_amdgcn_exp2f(fmaf(d, r.lo, fmaf(d, r.hi, -n))), (int)n);
  return d < r.least ? 0.f : e;  // (a NaN stays)
}

// Whether the pass over the row leaves the listed columns out
template <typename T, bool BUCKET>
constexpr bool kApart = BUCKET || sizeof(T) == 4;

// Sums of e^((x - m) scale) over some of a row's logits ({-infinity, 0} of nothing): a
// thread's in 32 bits, joined in 64.
struct Sum {
  float m;
  double s;
  __device__ __forceinline__ void raise(float to, const Rate& rate) {
    if (to == m) return;
    s = m == -INFINITY ? s : s * power<true>(m - to, rate);
    m = to;
  }
  __device__ __forceinline__ void join(Sum o, const Rate& rate) {
    const float to = fmaxf(m, o.m);
    raise(to, rate);
    o.raise(to, rate);
    s += o.s;
  }
};

struct LossArgs {
  int64_t ld, vocab;
  const float* top;
  int top_k;
  float scale;
  Rate rate;
  int splits;    // workgroups per row
  int64_t span;  // a split's columns (a multiple of a vector's)
  Sum* part;     // splits > 1: each one's sum
  float* loss;
  float* stats;
};

__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmax(v, __shfl_xor(v, off, 64));
  return v;
}

// Whether no entry before the i-th names its column
__device__ __forceinline__ bool first_of_its_column(const int32_t* column, int i) {
  const int32_t c = column[i];
  bool first = true;
  for (int j = 0; j < i; ++j) first &= column[j] != c;
  return first;
}

// Lane by lane whether no entry before names its column (entry 64 u + lane)
struct Firsts {
  bool of[kPerLane];
  __device__ __forceinline__ void find(const int32_t* column, int top_k) {
#pragma unroll
    for (int u = 0; u < kPerLane; ++u) {
      const int i = 64 * u + (threadIdx.x & 63);
      of[u] = i < top_k && first_of_its_column(column, i);
    }
  }
};

// The row's loss, by one wave: `a` is the sum over all of its columns, or (kApart) over those
// that are not listed.  `column`: the entries' columns, -1 where there is none.
template <typename T, bool BUCKET>
__device__ void put_loss(const LossArgs& g, const T* row, const int32_t* column, const Firsts& firsts,
                         int64_t r, const Sum& a) {
  const int lane = threadIdx.x & 63;
  constexpr bool APART = kApart<T, BUCKET>;
  const double scale = g.scale;
  double t[kPerLane], x[kPerLane];
  bool given[kPerLane];
  double tm = -INFINITY, xm = a.m;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    const int i = 64 * u + lane;
    const int32_t c = i < g.top_k ? column[i] : -1;
    given[u] = c >= 0;
    t[u] = given[u] ? (double)g.top[r * g.top_k + i] : -INFINITY;
    x[u] = given[u] ? (double)(float)row[c] : -INFINITY;
    tm = fmax(tm, t[u]);
    xm = fmax(xm, x[u]);
  }
  tm = BUCKET ? 0.0 : wave_max(tm);
  xm = APART ? wave_max(xm) : (double)a.m;
  // (a maximum passes over NaN: with 0 in its place the sum does not)
  bool odd = false;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) odd |= given[u] && t[u] != t[u];
  if (__any(odd)) tm = 0.0;
  // sums against xm: the listed columns' (each column once), and those of the rest
  double s = 0.0, p_sum = 0.0, p[kPerLane];
  const bool none = tm == -INFINITY;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    p[u] = 0.0;
    if (64 * u >= g.top_k) continue;
    p[u] = given[u] && !none ? exp(t[u] - tm) : 0.0;
    p_sum += p[u];
    if constexpr (APART) {
      if (given[u] && (x[u] > -INFINITY || x[u] != x[u]) && firsts.of[u]) s += exp((x[u] - xm) * scale);
    }
  }
  p_sum = wave_sum(p_sum);
  const double others = a.m == -INFINITY ? a.s : a.s * exp(((double)a.m - xm) * scale);
  s = APART ? wave_sum(s) + others : a.s;
  const double log_s = log(s), inv_p = BUCKET ? 1.0 : 1.0 / p_sum, log_p = BUCKET ? 0.0 : tm + log(p_sum);
  double loss = 0.0, weight = 0.0;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    if (64 * u >= g.top_k) continue;
    const double mass = none ? 0.0 : p[u] * inv_p;
    weight += mass;
    if (given[u] && mass != 0.0) {
      const double log_q = s == 0.0 ? -INFINITY : (x[u] - xm) * scale - log_s;
      loss += mass * (t[u] - log_p - log_q);
    }
  }
  loss = wave_sum(loss);
  weight = wave_sum(weight);
  // the gradient's factor of the columns that are not listed, against a.m
  const double beside = a.m == -INFINITY ? 0.0 : exp(((double)a.m - xm) * scale) / s;
  double rest_factor = weight * beside;
  if (BUCKET) {
    // (columns that are all masked, or none, are no bucket: what the rounding of the
    // teacher's values leaves of one less their sum would make the loss infinite.  Any that
    // is not masked makes one: q_r is taken by its logarithm, as it may be past a double.)
    const double p_r = 1.0 - weight;
    if (p_r > 0.0 && a.m > -INFINITY && a.s > 0.0) {
      const double log_r = ((double)a.m - xm) * scale + log(a.s) - log_s;
      loss += p_r * (log(p_r) - log_r);
      rest_factor = beside - p_r / a.s;
      weight = 1.0;
    } else if (others != others) {
      loss = others;
    }
  }
  if (lane == 0) {
    g.loss[r] = (float)loss;
    // what the gradient takes: at listed columns q_j = (stats[1] + [7]) e^((x_j - [0]) scale) with
    // the factor [2] and p_i = ([5] + [8]) e^(t_i - [4]), at others [3] e^((x_j - [9]) scale)
    float* o = g.stats + r * ISOLOCO_DISTILL_STATS;
    o[0] = s != s ? NAN : (float)xm;
    o[1] = (float)(1.0 / s);
    o[7] = s > 0.0 ? (float)(1.0 / s - (double)o[1]) : 0.f;
    o[2] = (float)weight;
    o[3] = (float)rest_factor;
    o[4] = none ? 0.f : (float)tm;
    o[5] = none ? 0.f : (float)inv_p;
    o[8] = none ? 0.f : (float)(inv_p - (double)o[5]);
    o[6] = s == 0.0 ? -INFINITY : (float)(xm * scale + log_s);
    // (columns that are all masked: 0 times what -infinity gives)
    o[9] = s != s ? NAN : a.m == -INFINITY ? 0.f : a.m;
  }
}

// a row without a teacher: no loss, and the gradient of nothing
__device__ __forceinline__ void put_none(const LossArgs& g, int64_t r) {
  g.loss[r] = 0.f;
  for (int i = 0; i < ISOLOCO_DISTILL_STATS; ++i) g.stats[r * ISOLOCO_DISTILL_STATS + i] = 0.f;
}

// The row's columns into `column`; whether there is any.
template <typename ID>
__device__ __forceinline__ bool load_columns(const ID* index, int64_t r, int top_k, int64_t vocab, int32_t* column) {
  bool any = false;
  for (int i = threadIdx.x; i < top_k; i += blockDim.x) {
    const int64_t c = index[r * top_k + i];
    const bool in = c >= 0 && c < vocab;
    column[i] = in ? (int32_t)c : -1;
    any |= in;
  }
  return __syncthreads_or(any);
}

// One workgroup of WAVES waves per row, or per split of a row: kHeld columns per thread at
// a time, as they are stored, their maximum and then their sum against it.
template <typename T, typename ID, int WAVES, bool BUCKET>
__global__ void __launch_bounds__(64 * WAVES, sizeof(T) == 2 ? 8 : 4)
    distill_kernel(const T* logits, const ID* index, LossArgs g) {
  constexpr int N = Vec<T>::N, kThreads = 64 * WAVES, kVecs = kHeld / N;
  constexpr int turn = kThreads * kVecs;  // vectors that the workgroup holds
  constexpr bool APART = kApart<T, BUCKET>;
  constexpr int kWords = !APART ? 1 : (WAVES == 8 ? (int)kMostSpan : WAVES == 4 ? kHalfTurns * turn * N : turn * N) / 32;
  __shared__ Sum part[WAVES];
  __shared__ int32_t column[ISOLOCO_MAX_TEACHER];
  __shared__ uint32_t marks[kWords];
  const int64_t r = blockIdx.x / g.splits;
  const int split = (int)(blockIdx.x - r * g.splits);
  const int64_t begin = split * g.span;
  const int count = (int)min(g.span, g.vocab - begin), whole = count / N;
  const T* row = logits + r * g.ld;
  const T* p = row + begin;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  u32x4 v[kVecs];
  float last;
  const auto load = [&](int base) {
#pragma unroll
    for (int c = 0; c < kVecs; ++c) {
      const int i = base + c * kThreads + (int)threadIdx.x;
      v[c] = sizeof(T) == 2 ? (u32x4)(0xff80ff80u) : (u32x4)(0xff800000u);  // -infinity
      if (i < whole) v[c] = *reinterpret_cast<const u32x4_any*>(p + (int64_t)i * N);
    }
    const int at = whole * N + (int)threadIdx.x;
    last = base == 0 && at < count ? (float)p[at] : -INFINITY;
  };
  if constexpr (APART) {
    for (int i = threadIdx.x; i < (count + 31) / 32; i += kThreads) marks[i] = 0;
  }
  const bool any = load_columns(index, r, g.top_k, g.vocab, column);
  if (!any) {
    if (split == 0 && threadIdx.x == 0) put_none(g, r);
    return;
  }
  if constexpr (APART) {
    for (int i = threadIdx.x; i < g.top_k; i += kThreads) {
      const int64_t c = column[i] - begin;
      if (column[i] >= 0 && c >= 0 && c < count) atomicOr(&marks[c >> 5], 1u << (c & 31));
    }
    __syncthreads();
  }

  struct {
    float m, s;
  } own = {-INFINITY, 0.f};
  load(0);
  // (while the first of them come)
  Firsts firsts;
  if constexpr (APART) {
    if (wave == 0) firsts.find(column, g.top_k);
  }
  for (int base = 0; base == 0 || base < whole; base += turn) {
    if (base) load(base);
    if constexpr (APART) {
#pragma unroll
      for (int c = 0; c < kVecs; ++c) {
        const int i = base + c * kThreads + (int)threadIdx.x;
        if (i < whole) {
          uint32_t bits = reinterpret_cast<const uint8_t*>(marks)[i * N / 8];
          if (N == 4) bits = (bits >> (4 * (i & 1))) & 15u;
          if (bits) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if constexpr (N == 4) {
                if (bits >> w & 1u) v[c][w] = 0xff800000u;
              } else {
                if (bits >> (2 * w) & 1u) v[c][w] = (v[c][w] & 0xffff0000u) | 0xff80u;
                if (bits >> (2 * w + 1) & 1u) v[c][w] = (v[c][w] & 0xffffu) | 0xff800000u;
              }
            }
          }
        }
      }
      const int at = whole * N + (int)threadIdx.x;
      if (at < count && (marks[at >> 5] >> (at & 31) & 1u)) last = -INFINITY;
    }
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
    most = fmaxf(own.m, most);
    if (most != own.m && own.m != -INFINITY) own.s *= power<true>(own.m - most, g.rate);
    own.m = most;
    const float m = most == -INFINITY ? 0.f : most;
#pragma unroll
    for (int c = 0; c < kVecs; ++c)
      if (base + c * kThreads < whole) {
        float x[N];
        unpack<T>(v[c], x);
#pragma unroll
        for (int e = 0; e < N; ++e) own.s += power<sizeof(T) == 4>(x[e] - m, g.rate);
      }
    if (base == 0) own.s += power<sizeof(T) == 4>(last - m, g.rate);
  }
  Sum a = {own.m, own.s};
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    Sum o;
    o.m = __shfl_xor(a.m, off, 64);
    o.s = __shfl_xor(a.s, off, 64);
    a.join(o, g.rate);
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) part[wave] = a;
    __syncthreads();
    a = part[0];
    for (int w = 1; w < WAVES; ++w) a.join(part[w], g.rate);
  }
  if (wave > 0) return;
  if (g.splits > 1) {
    if (lane == 0) g.part[blockIdx.x] = a;
  } else {
    put_loss<T, BUCKET>(g, row, column, firsts, r, a);
  }
}

// A row's splits joined, in their order, by one wave.
template <typename T, typename ID, bool BUCKET>
__global__ void __launch_bounds__(64) distill_join_kernel(const T* logits, const ID* index, LossArgs g) {
  __shared__ int32_t column[ISOLOCO_MAX_TEACHER];
  const int64_t r = blockIdx.x;
  if (!load_columns(index, r, g.top_k, g.vocab, column)) return;  // (put_none is done)
  const Sum* part = g.part + r * g.splits;
  Sum a = part[0];
  for (int i = 1; i < g.splits; ++i) a.join(part[i], g.rate);
  Firsts firsts;
  if constexpr (kApart<T, BUCKET>) firsts.find(column, g.top_k);
  put_loss<T, BUCKET>(g, logits + r * g.ld, column, firsts, r, a);
}

struct GradArgs {
  int64_t ld, rows, vocab, ld_d;
  const float* top;
  int top_k;
  float scale;
  Rate rate;
  const float* stats;
  const float* dloss;
  int spans;
};

constexpr int kGradThreads = 256;
constexpr int kGradVecs = 4;  // 16-byte vectors of a thread

// One workgroup per row and span of kGradThreads * kGradVecs vectors: every column as one
// that is not listed, then the listed ones over them (their logits are read before: the
// result may lie over the logits).  PAST: the result goes past the caches.
template <typename T, typename ID, bool PAST>
__global__ void __launch_bounds__(kGradThreads) distill_grad_kernel(const T* logits, const ID* index, T* dlogits,
                                                                    GradArgs g) {
  constexpr int N = Vec<T>::N;
  __shared__ int32_t column[ISOLOCO_MAX_TEACHER];
  // q and p are near each other once the student has learnt: float32 results take their
  // difference in 64 bits
  typedef typename std::conditional<sizeof(T) == 4, double, float>::type Fine;
  __shared__ Fine mass[ISOLOCO_MAX_TEACHER];
  static_assert(ISOLOCO_MAX_TEACHER <= kGradThreads, "one entry a thread");
  // (the last rows first: the forward pass read them last, some are still in a cache)
  const int64_t r = g.rows - 1 - blockIdx.x / g.spans;
  const int span = (int)(blockIdx.x % g.spans);
  const int64_t first = (int64_t)span * (kGradThreads * kGradVecs), whole = g.vocab / N;
  const T* row = logits + r * g.ld;
  T* out = dlogits + r * g.ld_d;
  const float* st = g.stats + r * ISOLOCO_DISTILL_STATS;
  const float m = st[0], inv_s = st[1], factor = st[2], tm = st[4], inv_p = st[5];
  const float dl = g.dloss[r] * g.scale;
  // nothing to hand back: no loss wanted, no teacher, no student
  const bool none = dl == 0.f || inv_p == 0.f || m == -INFINITY;
  const float from = none ? 0.f : m, from_other = st[9];
  u32x4 v[kGradVecs];
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int64_t i = first + u * kGradThreads + threadIdx.x;
    v[u] = (u32x4){};
    if (!none && i < whole) v[u] = *reinterpret_cast<const u32x4_any*>(row + i * N);
  }
  const int64_t at = whole * N + threadIdx.x;
  const bool single = span == 0 && at < g.vocab;
  const float end = single && !none ? (float)row[at] : 0.f;
  // this thread's entry, if its column is of this span
  const int i = threadIdx.x;
  bool mine = false;
  int64_t c = -1;
  float x_top = 0.f;
  if (!none && i < g.top_k) {
    c = index[r * g.top_k + i];
    const bool in = c >= 0 && c < g.vocab;
    column[i] = in ? (int32_t)c : -1;
    if constexpr (sizeof(T) == 4)
      mass[i] = in ? ((double)inv_p + (double)st[8]) * exp((double)g.top[r * g.top_k + i] - (double)tm) : 0.0;
    else
      mass[i] = in ? inv_p * expf(g.top[r * g.top_k + i] - tm) : 0.f;
    const int64_t vec = c / N;
    mine = in && (vec >= whole ? span == 0 : vec >= first && vec < first + kGradThreads * kGradVecs);
    if (mine) x_top = (float)row[c];
  }
  __syncthreads();
  const float other = none ? 0.f : st[3] * dl;
  const auto grad = [&](float x) { return none ? 0.f : power<sizeof(T) == 4>(x - from_other, g.rate) * other; };
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int64_t j = first + u * kGradThreads + threadIdx.x;
    if (j < whole) {
      float x[N];
      unpack<T>(v[u], x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = grad(x[e]);
      const u32x4 d = pack<T>(x);
      u32x4_any* to = reinterpret_cast<u32x4_any*>(out + j * N);
      if constexpr (PAST) __builtin_nontemporal_store(d, to);
      else *to = d;
    }
  }
  if (single) out[at] = (T)grad(end);
  if (none) return;
  // every wave's stores are done before the listed columns' go over them
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (!mine || !first_of_its_column(column, i)) return;
  Fine p = 0, q;
  for (int j = i; j < g.top_k; ++j) p += column[j] == (int32_t)c ? mass[j] : (Fine)0;
  if constexpr (sizeof(T) == 4)
    q = exp(((double)x_top - (double)from) * (double)g.scale) * ((double)inv_s + (double)st[7]);
  else
    q = power<true>(x_top - from, g.rate) * inv_s;
  out[c] = (T)(float)((q * factor - p) * dl);
}

struct DistillShape {
  int64_t rows, vocab;
  int32_t dtype, index_type, top_k, rest;
  float scale;
};

isoloco_status check_shape(const DistillShape& s) {
  if (s.rows < 0 || s.rows > kMaxExtent / 2 || s.vocab < 1 || s.vocab > kMaxExtent / 2)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld rows of %lld logits", (long long)s.rows, (long long)s.vocab);
  if (!is_dtype(s.dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", s.dtype);
  if (!is_index_type(s.index_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "index type %d", s.index_type);
  if (s.top_k < 1 || s.top_k > ISOLOCO_MAX_TEACHER)
    return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d, of 1 to %d", s.top_k, ISOLOCO_MAX_TEACHER);
  if (s.rest != ISOLOCO_REST_DROP && s.rest != ISOLOCO_REST_BUCKET) return fail(ISOLOCO_ERR_INVALID_ARG, "rest %d", s.rest);
  if (!(s.scale > 0.f) || isinf(s.scale))
    return fail(ISOLOCO_ERR_INVALID_ARG, "scale = %g: a positive number is wanted", (double)s.scale);
  return ISOLOCO_OK;
}

// Workgroups per row: one, unless the rows are few and long, or longer than a bitmap.  Both sides
// measured, us a call of a graph with the rest in bfloat16, 1 / 2 / 4 / 8 / 16 splits:
//            1 row                              127 rows                           256 rows
//    32000   9.5 / 11.8 / 11.1 / 11.7 / 12.6    10.1 / 12.4 / 12.5 / 12.8 / 14.4   10.4 / 13.5 / 14.4 / 14.0 / 16.4
//    50257   11.3 / 11.8 / 11.6 / 11.7 / 13.1   13.2 / 13.5 / 13.6 / 14.8 / 15.5   13.6 / 17.1 / 17.2 / 19.8 / 18.8
//   128000   16.7 / 14.7 / 12.3 / 12.2 / 13.2   18.3 / 17.1 / 17.3 / 17.7 / 21.3   20.9 / 23.7 / 23.3 / 24.3 / 29.7
int splits_of(int64_t rows, int64_t vocab) {
  int64_t s = 1;
  if (rows < 128 && vocab > 80000) {
    const int64_t most = vocab / 24576, wanted = 512 / (rows ? rows : 1);
    s = most < wanted ? most : wanted;
    s = s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s;
  }
  const int64_t least = (vocab + kMostSpan - 8) / (kMostSpan - 7);
  return (int)(s > least ? s : least);
}

size_t distill_workspace(int64_t rows, int64_t vocab) {
  const size_t s = (size_t)splits_of(rows, vocab);
  return s > 1 ? (size_t)rows * s * sizeof(Sum) : 0;
}

// One wave if it holds the row (or split) at once, 256 threads if they do in two turns.  (8192
// rows of 32000, us, in 512 threads' one turn / 256 threads' two: 115 / 98.9 in bfloat16, 137 /
// 117 with the rest; 192 / 193 and 226 / 192 in float32.  4096 rows of 128000 in four / eight: 198
// / 214 in bfloat16 with the rest, 366 / 375 in float32.)
int threads_of(int64_t span, int64_t blocks) {
  if (span <= 64 * kHeld) return 64;
  // (up to two workgroups a CU: the shorter way for each; 16 rows of 32000 in 256 / 512 threads
  // 12.2 / 11.1 us in bfloat16, 15.2 / 13.4 in float32)
  return span <= 256 * kHeld || (span <= kHalfTurns * 256 * kHeld && blocks > 512) ? 256 : 512;
}

template <typename T, typename ID, bool BUCKET>
void run_loss(const T* l, const ID* index, int64_t rows, const LossArgs& g, hipStream_t st) {
  const dim3 grid((unsigned)(rows * g.splits));
  const int threads = threads_of(g.span, rows * g.splits);
  if (threads == 64) hipLaunchKernelGGL((distill_kernel<T, ID, 1, BUCKET>), grid, dim3(64), 0, st, l, index, g);
  else if (threads == 256) hipLaunchKernelGGL((distill_kernel<T, ID, 4, BUCKET>), grid, dim3(256), 0, st, l, index, g);
  else hipLaunchKernelGGL((distill_kernel<T, ID, 8, BUCKET>), grid, dim3(512), 0, st, l, index, g);
  if (g.splits > 1)
    hipLaunchKernelGGL((distill_join_kernel<T, ID, BUCKET>), dim3((unsigned)rows), dim3(64), 0, st, l, index, g);
}

template <typename T, typename ID>
void run_forward(const void* logits, const void* index, int64_t rows, int rest, const LossArgs& g, hipStream_t st) {
  const T* l = static_cast<const T*>(logits);
  const ID* i = static_cast<const ID*>(index);
  if (rest == ISOLOCO_REST_BUCKET) run_loss<T, ID, true>(l, i, rows, g, st);
  else run_loss<T, ID, false>(l, i, rows, g, st);
}

template <typename T, typename ID>
void run_grad(const void* logits, const void* index, void* dlogits, const GradArgs& g, hipStream_t st) {
  const bool past = dlogits != logits && g.rows * g.vocab * (int64_t)sizeof(T) > kCacheBytes;
  hipLaunchKernelGGL((past ? distill_grad_kernel<T, ID, true> : distill_grad_kernel<T, ID, false>),
                     dim3((unsigned)(g.rows * g.spans)), dim3(kGradThreads), 0, st, static_cast<const T*>(logits),
                     static_cast<const ID*>(index), static_cast<T*>(dlogits), g);
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

#define BY_TYPES(RUN, ...)                                                             \
  do {                                                                                 \
    if (dtype == ISOLOCO_F32) {                                                        \
      if (index_type == ISOLOCO_I32) RUN<float, int32_t>(__VA_ARGS__);                 \
      else RUN<float, int64_t>(__VA_ARGS__);                                           \
    } else {                                                                           \
      if (index_type == ISOLOCO_I32) RUN<__bf16, int32_t>(__VA_ARGS__);                \
      else RUN<__bf16, int64_t>(__VA_ARGS__);                                          \
    }                                                                                  \
  } while (0)

extern "C" {

isoloco_status isoloco_distill_loss_workspace_size(int64_t rows, int64_t vocab, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  ISOLOCO_TRY(check_shape({rows, vocab, ISOLOCO_F32, ISOLOCO_I32, 1, ISOLOCO_REST_DROP, 1.f}));
  *bytes = distill_workspace(rows, vocab);
  return ISOLOCO_OK;
}

isoloco_status isoloco_distill_loss(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows, int64_t vocab,
                                    const float* top_logprob, const void* top_index, int32_t index_type, int32_t top_k,
                                    float scale, int32_t rest, float* loss, float* stats, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  ISOLOCO_TRY(check_shape({rows, vocab, dtype, index_type, top_k, rest, scale}));
  if (rows == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type), n = (size_t)rows * top_k;
  ISOLOCO_TRY(check_matrix("logits", logits, rows, vocab, ld_logits, e));
  const size_t need = distill_workspace(rows, vocab);
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const Operand ins[] = {{"logits", logits, matrix_bytes(rows, vocab, ld_logits, e), e},
                         {"top_logprob", top_logprob, n * 4, 4},
                         {"top_index", top_index, n * ib, ib}};
  const Operand outs[] = {{"loss", loss, (size_t)rows * 4, 4},
                          {"stats", stats, (size_t)rows * 4 * ISOLOCO_DISTILL_STATS, 4},
                          {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_operands(outs, 3, ins, 3));
  LossArgs g;
  g.ld = ld_logits;
  g.vocab = vocab;
  g.top = top_logprob;
  g.top_k = top_k;
  g.scale = scale;
  g.rate = rate_parts(scale);
  g.splits = splits_of(rows, vocab);
  g.span = ((vocab + g.splits - 1) / g.splits + 7) / 8 * 8;
  g.splits = (int)((vocab + g.span - 1) / g.span);
  g.part = static_cast<Sum*>(workspace);
  g.loss = loss;
  g.stats = stats;
  if (!launchable(rows * g.splits, threads_of(g.span, rows * g.splits)))
    return fail(ISOLOCO_ERR_UNSUPPORTED, "too many rows for one launch");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_forward, logits, top_index, rows, rest, g, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "distillation loss");
}

isoloco_status isoloco_distill_loss_backward(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                             int64_t vocab, const float* top_logprob, const void* top_index,
                                             int32_t index_type, int32_t top_k, float scale, int32_t rest,
                                             const float* stats, const float* dloss, void* dlogits, int64_t ld_dlogits,
                                             void* hip_stream) {
  ISOLOCO_TRY(check_shape({rows, vocab, dtype, index_type, top_k, rest, scale}));
  if (rows == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), ib = index_bytes(index_type), n = (size_t)rows * top_k;
  ISOLOCO_TRY(check_matrix("logits", logits, rows, vocab, ld_logits, e));
  ISOLOCO_TRY(check_matrix("dlogits", dlogits, rows, vocab, ld_dlogits, e));
  // in place: every element is read before it is written
  const bool in_place = dlogits == logits && ld_dlogits == ld_logits;
  const Operand ins[] = {{"top_logprob", top_logprob, n * 4, 4},
                         {"top_index", top_index, n * ib, ib},
                         {"stats", stats, (size_t)rows * 4 * ISOLOCO_DISTILL_STATS, 4},
                         {"dloss", dloss, (size_t)rows * 4, 4},
                         {"the logits", logits, in_place ? 0 : matrix_bytes(rows, vocab, ld_logits, e), e}};
  const Operand outs[] = {{"dlogits", dlogits, matrix_bytes(rows, vocab, ld_dlogits, e), e}};
  ISOLOCO_TRY(check_operands(outs, 1, ins, 5));
  const int64_t vecs = vocab / (16 / (int64_t)e);
  const int64_t spans = vecs == 0 ? 1 : (vecs + kGradThreads * kGradVecs - 1) / (kGradThreads * kGradVecs);
  if (!launchable(rows * spans, kGradThreads)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  GradArgs g;
  g.ld = ld_logits;
  g.rows = rows;
  g.vocab = vocab;
  g.ld_d = ld_dlogits;
  g.top = top_logprob;
  g.top_k = top_k;
  g.scale = scale;
  g.rate = rate_parts(scale);
  g.stats = stats;
  g.dloss = dloss;
  g.spans = (int)spans;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  BY_TYPES(run_grad, logits, top_index, dlogits, g, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "gradient of the distillation loss");
}

}  // extern "C"
