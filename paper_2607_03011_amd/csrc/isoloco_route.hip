// Routing of tokens to experts, and the grouping of the rows that the experts work on.
// With x the scores of a token and p their softmax:
//
//   the top_k largest scores (of equal ones the lower expert first), expert_j
//   weight_j = p_j, or (normalize) p_j over their sum: the softmax of the chosen scores
//
// The slots (token, j) are then put in the order of their experts, and of the slots within
// an expert: offsets[e] is where expert e's begin, row[token, j] the place of a slot, and
// token[r] the token of place r.  A score of -infinity is no expert to choose: a slot that
// finds none has expert -1 and weight 0, and stands behind the last expert's.
//
//   gradient, g_j that of weight_j:  normalize  dx_j = w_j (g_j - sum_i w_i g_i), 0 elsewhere
//                                    otherwise  dx_e = p_e (sum of the g_j at e - sum_i w_i g_i)
//
// No atomics decide an order: a workgroup counts its slots by expert, and the next launch's
// workgroup of the same slots adds up the counts before its own and ranks its slots by wave.
// Bounded by latency: the scores of 16384 tokens are a few MB; the choosing is top_k rounds of a
// maximum over a wave, which stays in the vector registers (over LDS, and with a launch of its
// own for the sums of counts, the three launches for 16384 tokens of 64 experts took 65 us).
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSmallTokens = 64;  // so many are routed by one workgroup
constexpr int kMostBlocks = 256;  // each adds up the counts of all

struct RouteArgs {
  int64_t ld, tokens;
  int experts, top_k, normalize;
  float* weight;
  int32_t *expert, *row, *token, *offsets;
  int32_t* counts;  // workgroups x (experts + 1)
  int per_block;    // tokens of a workgroup
  int blocks;
};

// Over the lanes up to each: within rows of 16, then a row's last to the next, then two rows'
// to the other two; lane 63 has all.
template <typename F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, const F& join) {
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = join(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}
__device__ __forceinline__ uint32_t max_of(uint32_t v) {
  return __builtin_amdgcn_readlane(over_lanes(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63);
}
__device__ __forceinline__ float sum_of(float v) {
  return __uint_as_float(__builtin_amdgcn_readlane(
      over_lanes(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }),
      63));
}
__device__ __forceinline__ int scan_of(int v) {
  return (int)over_lanes((uint32_t)v, [](uint32_t a, uint32_t b) { return a + b; });
}

// One wave chooses a token's experts: lane j gets the j-th (-1: none), and its weight.
template <typename T, int EL>
__device__ __forceinline__ void choose(const T* scores, const RouteArgs& g, int& expert, float& weight) {
  const int lane = threadIdx.x & 63;
  uint32_t key[EL];  // the order of the values; 0: chosen, or no expert
  float x[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = 64 * i + lane;
    x[i] = e < g.experts ? (float)scores[e] : -INFINITY;
    key[i] = e < g.experts ? order_of(x[i]) : 0;
  }
  uint32_t mine = 0;
  expert = -1;
  for (int j = 0; j < g.top_k; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) best = key[i] > best ? key[i] : best;
    best = max_of(best);
    // the lowest expert that has it
    bool found = false;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const uint64_t at = __ballot(key[i] == best);
      if (!found && at) {
        found = true;
        const int winner = __ffsll((unsigned long long)at) - 1;
        if (lane == winner) key[i] = 0;
        if (lane == j) {
          mine = best;
          expert = 64 * i + winner;
        }
      }
    }
  }
  const float value = lane < g.top_k ? value_of((uint64_t)mine << 32) : -INFINITY;
  const float m = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(value), 0));
  if (value == -INFINITY) expert = -1;
  const float e = value == -INFINITY ? 0.f : expf(value - m);
  float s = e;
  if (!g.normalize) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) s += x[i] == -INFINITY ? 0.f : expf(x[i] - m);
  }
  s = sum_of(s);
  weight = expert < 0 ? 0.f : e / s;
}

// The workgroup's tokens: their experts and weights, and the slots' counts by group (of which
// the last is no expert).
template <typename T, int EL>
__device__ __forceinline__ void choose_all(const T* scores, const RouteArgs& g, int64_t first, int64_t end, int32_t* count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i <= g.experts; i += kThreads) count[i] = 0;
  __syncthreads();
  for (int64_t t = first + wave; t < end; t += kWaves) {
    int expert;
    float weight;
    choose<T, EL>(scores + t * g.ld, g, expert, weight);
    if (lane < g.top_k) {
      const int64_t slot = t * g.top_k + lane;
      g.weight[slot] = weight;
      g.expert[slot] = expert;
      atomicAdd(&count[expert < 0 ? g.experts : expert], 1);
    }
  }
  __syncthreads();
}

// The scan of `total` over the groups, in place, by one wave.
__device__ __forceinline__ void scan_groups(int32_t* total, int groups) {
  const int lane = threadIdx.x & 63;
  int carry = 0;
  for (int base = 0; base < groups; base += 64) {
    const int i = base + lane, n = i < groups ? total[i] : 0, upto = scan_of(n);
    if (i < groups) total[i] = carry + upto - n;
    carry += __builtin_amdgcn_readlane(upto, 63);
  }
}

// The workgroup places its slots in their order; next[i] is the place of group i's next one.
__device__ __forceinline__ void place(const RouteArgs& g, int64_t first, int64_t end, int32_t* next,
                                      uint8_t (*of_wave)[ISOLOCO_MAX_EXPERTS + 4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = g.experts + 1;
  int bits = 0;
  while ((1 << bits) < groups) ++bits;
  for (int64_t base = first; base < end; base += kThreads) {
    for (int i = threadIdx.x; i < kWaves * (ISOLOCO_MAX_EXPERTS + 4) / 4; i += kThreads)
      reinterpret_cast<uint32_t*>(of_wave)[i] = 0;
    __syncthreads();
    const int64_t slot = base + threadIdx.x;
    const bool live = slot < end;
    int group = live ? g.expert[slot] : 0;
    if (group < 0) group = g.experts;
    // the wave's lanes of the same group
    uint64_t same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(group >> b & 1);
      same &= group >> b & 1 ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << lane) - 1));
    if (live && (same >> lane) == 1) of_wave[wave][group] = (uint8_t)(before + 1);
    __syncthreads();
    if (live) {
      int at = next[group] + before;
      for (int w = 0; w < wave; ++w) at += of_wave[w][group];
      g.row[slot] = at;
      g.token[at] = (int32_t)(slot / g.top_k);
    }
    if (base + kThreads >= end) return;
    __syncthreads();
    for (int i = threadIdx.x; i < groups; i += kThreads) {
      int sum = 0;
      for (int w = 0; w < kWaves; ++w) sum += of_wave[w][i];
      next[i] += sum;
    }
    __syncthreads();
  }
}

// Everything, by one workgroup.
template <typename T, int EL>
__global__ void __launch_bounds__(kThreads) route_small_kernel(const T* scores, RouteArgs g) {
  __shared__ int32_t next[ISOLOCO_MAX_EXPERTS + 1];
  __shared__ __attribute__((aligned(4))) uint8_t of_wave[kWaves][ISOLOCO_MAX_EXPERTS + 4];
  choose_all<T, EL>(scores, g, 0, g.tokens, next);
  if (threadIdx.x < 64) scan_groups(next, g.experts + 1);
  __syncthreads();  // (the experts that were stored are read again, too)
  for (int i = threadIdx.x; i <= g.experts; i += kThreads) g.offsets[i] = next[i];
  place(g, 0, g.tokens * g.top_k, next, of_wave);
}

// The choice of a workgroup's tokens, and its slots' counts.
template <typename T, int EL>
__global__ void __launch_bounds__(kThreads) route_choose_kernel(const T* scores, RouteArgs g) {
  __shared__ int32_t count[ISOLOCO_MAX_EXPERTS + 1];
  const int64_t first = (int64_t)blockIdx.x * g.per_block, end = min(g.tokens, first + g.per_block);
  choose_all<T, EL>(scores, g, first, end, count);
  int32_t* out = g.counts + (int64_t)blockIdx.x * (g.experts + 1);
  for (int i = threadIdx.x; i <= g.experts; i += kThreads) out[i] = count[i];
}

// The places of the same workgroup's slots: 64 groups at a time, each wave adds up some of the
// workgroups' counts, those before this one apart.
__global__ void __launch_bounds__(kThreads) route_place_kernel(RouteArgs g) {
  __shared__ int32_t next[ISOLOCO_MAX_EXPERTS + 1], earlier[ISOLOCO_MAX_EXPERTS + 1];
  __shared__ int32_t sum[kWaves][64], sum_before[kWaves][64];
  __shared__ __attribute__((aligned(4))) uint8_t of_wave[kWaves][ISOLOCO_MAX_EXPERTS + 4];
  constexpr int kPer = kMostBlocks / kWaves;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = g.experts + 1;
  for (int base = 0; base < groups; base += 64) {
    int n[kPer], all = 0, before = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int b = wave * kPer + u;
      n[u] = b < g.blocks && base + lane < groups ? g.counts[(int64_t)b * groups + base + lane] : 0;
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      all += n[u];
      before += wave * kPer + u < (int)blockIdx.x ? n[u] : 0;
    }
    sum[wave][lane] = all;
    sum_before[wave][lane] = before;
    __syncthreads();
    if (wave < 2 && base + lane < groups) {
      int s = 0;
      for (int w = 0; w < kWaves; ++w) s += wave ? sum_before[w][lane] : sum[w][lane];
      (wave ? earlier : next)[base + lane] = s;
    }
    __syncthreads();
  }
  if (wave == 0) scan_groups(next, groups);
  __syncthreads();
  for (int i = threadIdx.x; i < groups; i += kThreads) {
    if (blockIdx.x == 0) g.offsets[i] = next[i];
    next[i] += earlier[i];
  }
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * g.per_block, end = min(g.tokens, first + g.per_block);
  place(g, first * g.top_k, end * g.top_k, next, of_wave);
}

struct RouteGradArgs {
  int64_t ld, tokens, ld_d;
  int experts, top_k, normalize;
  const int32_t* expert;
  const float* dweight;
};

// One wave per token.
template <typename T, int EL>
__global__ void __launch_bounds__(256) route_grad_kernel(const T* scores, T* dscores, RouteGradArgs g) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= g.tokens) return;
  const T* row = scores + t * g.ld;
  float x[EL], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = 64 * i + lane;
    x[i] = e < g.experts ? (float)row[e] : -INFINITY;
  }
  // lane j: the j-th choice
  int expert = lane < g.top_k ? g.expert[t * g.top_k + lane] : -1;
  if (expert >= g.experts) expert = -1;
  const float chosen = expert < 0 ? -INFINITY : (float)row[expert];
  const float grad = expert < 0 ? 0.f : g.dweight[t * g.top_k + lane];
  if (g.normalize) {
    m = chosen;
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) m = fmaxf(m, x[i]);
  }
  m = value_of((uint64_t)max_of(order_of(m)) << 32);
  const float from = m == -INFINITY ? 0.f : m;
  float p[EL], s = 0.f, w = expert < 0 ? 0.f : expf(chosen - from);
  if (g.normalize) {
    s = w;
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      p[i] = expf(x[i] - from);
      s += p[i];
    }
  }
  s = sum_of(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
  w *= inv;
  const float inner = sum_of(w * grad);
  float d[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) d[i] = g.normalize ? 0.f : -(p[i] * inv) * inner;
  const float own = w * (g.normalize ? grad - inner : grad);
  for (int j = 0; j < g.top_k; ++j) {
    const int e = __builtin_amdgcn_readlane(expert, j);
    const float v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own), j));
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (e == 64 * i + lane) d[i] += v;
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = 64 * i + lane;
    if (e < g.experts) dscores[t * g.ld_d + e] = (T)d[i];
  }
}

isoloco_status check_shape(int64_t tokens, int64_t experts, int32_t top_k, int32_t dtype) {
  if (experts < 1 || experts > ISOLOCO_MAX_EXPERTS)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld experts, of 1 to %d", (long long)experts, ISOLOCO_MAX_EXPERTS);
  if (top_k < 1 || top_k > ISOLOCO_MAX_TOP || top_k > experts)
    return fail(ISOLOCO_ERR_INVALID_ARG, "top_k = %d of %lld, at most %d", top_k, (long long)experts, ISOLOCO_MAX_TOP);
  // (rows are counted in 31 bits)
  if (tokens < 0 || tokens > (kMaxExtent - 1) / top_k)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%lld tokens of %d experts", (long long)tokens, top_k);
  if (!is_dtype(dtype)) return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d", dtype);
  return ISOLOCO_OK;
}

// Tokens of a workgroup: 64, or more where that makes too many workgroups.
int64_t per_block_of(int64_t tokens) {
  return std::max<int64_t>(64, (tokens + kMostBlocks - 1) / kMostBlocks);
}

size_t route_workspace(int64_t tokens, int64_t experts) {
  if (tokens <= kSmallTokens) return 0;
  const int64_t per = per_block_of(tokens);
  return (size_t)((tokens + per - 1) / per) * (size_t)(experts + 1) * 4;
}

template <typename T, int EL>
void run_forward(const void* scores, const RouteArgs& g, hipStream_t st) {
  const T* s = static_cast<const T*>(scores);
  if (g.tokens <= kSmallTokens) {
    hipLaunchKernelGGL((route_small_kernel<T, EL>), dim3(1), dim3(kThreads), 0, st, s, g);
    return;
  }
  hipLaunchKernelGGL((route_choose_kernel<T, EL>), dim3(g.blocks), dim3(kThreads), 0, st, s, g);
  hipLaunchKernelGGL(route_place_kernel, dim3(g.blocks), dim3(kThreads), 0, st, g);
}

template <typename T, int EL>
void run_grad(const void* scores, void* dscores, const RouteGradArgs& g, hipStream_t st) {
  hipLaunchKernelGGL((route_grad_kernel<T, EL>), dim3((unsigned)((g.tokens + 3) / 4)), dim3(256), 0, st,
                     static_cast<const T*>(scores), static_cast<T*>(dscores), g);
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

#define BY_EXPERTS(RUN, T, ...)                           \
  do {                                                    \
    if (experts <= 64) RUN<T, 1>(__VA_ARGS__);            \
    else if (experts <= 128) RUN<T, 2>(__VA_ARGS__);      \
    else if (experts <= 256) RUN<T, 4>(__VA_ARGS__);      \
    else if (experts <= 512) RUN<T, 8>(__VA_ARGS__);      \
    else RUN<T, 16>(__VA_ARGS__);                         \
  } while (0)

extern "C" {

isoloco_status isoloco_route_tokens_workspace_size(int64_t tokens, int64_t experts, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  ISOLOCO_TRY(check_shape(tokens, experts, 1, ISOLOCO_F32));
  *bytes = route_workspace(tokens, experts);
  return ISOLOCO_OK;
}

isoloco_status isoloco_route_tokens(const void* scores, int64_t ld_scores, int32_t dtype, int64_t tokens,
                                    int64_t experts, int32_t top_k, int32_t normalize, float* weight, int32_t* expert,
                                    int32_t* row, int32_t* token, int32_t* offsets, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  ISOLOCO_TRY(check_shape(tokens, experts, top_k, dtype));
  const size_t e = dtype_bytes(dtype), n = (size_t)tokens * top_k * 4, need = route_workspace(tokens, experts);
  ISOLOCO_TRY(check_matrix("scores", scores, tokens, experts, ld_scores, e));
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const Operand ins[] = {{"scores", scores, matrix_bytes(tokens, experts, ld_scores, e), e}};
  const Operand outs[] = {{"weight", weight, n, 4}, {"expert", expert, n, 4}, {"row", row, n, 4}, {"token", token, n, 4},
                          {"offsets", offsets, (size_t)(experts + 1) * 4, 4}, {"the workspace", workspace, need, 1}};
  ISOLOCO_TRY(check_operands(outs, 6, ins, 1));
  RouteArgs g;
  g.ld = ld_scores;
  g.tokens = tokens;
  g.experts = (int)experts;
  g.top_k = top_k;
  g.normalize = normalize != 0;
  g.weight = weight;
  g.expert = expert;
  g.row = row;
  g.token = token;
  g.offsets = offsets;
  g.per_block = (int)per_block_of(tokens);
  g.blocks = (int)((tokens + g.per_block - 1) / g.per_block);
  g.counts = static_cast<int32_t*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == ISOLOCO_F32) BY_EXPERTS(run_forward, float, scores, g, st);
  else BY_EXPERTS(run_forward, __bf16, scores, g, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "routing of tokens");
}

isoloco_status isoloco_route_tokens_backward(const void* scores, int64_t ld_scores, int32_t dtype, int64_t tokens,
                                             int64_t experts, int32_t top_k, int32_t normalize, const int32_t* expert,
                                             const float* dweight, void* dscores, int64_t ld_dscores,
                                             void* hip_stream) {
  ISOLOCO_TRY(check_shape(tokens, experts, top_k, dtype));
  if (tokens == 0) return ISOLOCO_OK;
  const size_t e = dtype_bytes(dtype), n = (size_t)tokens * top_k * 4;
  ISOLOCO_TRY(check_matrix("scores", scores, tokens, experts, ld_scores, e));
  ISOLOCO_TRY(check_matrix("dscores", dscores, tokens, experts, ld_dscores, e));
  const Operand ins[] = {{"scores", scores, matrix_bytes(tokens, experts, ld_scores, e), e},
                         {"expert", expert, n, 4},
                         {"dweight", dweight, n, 4}};
  const Operand outs[] = {{"dscores", dscores, matrix_bytes(tokens, experts, ld_dscores, e), e}};
  ISOLOCO_TRY(check_operands(outs, 1, ins, 3));
  if (!launchable((tokens + 3) / 4, 256)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many tokens for one launch");
  const RouteGradArgs g = {ld_scores, tokens, ld_dscores, (int)experts, top_k, normalize != 0, expert, dweight};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == ISOLOCO_F32) BY_EXPERTS(run_grad, float, scores, dscores, g, st);
  else BY_EXPERTS(run_grad, __bf16, scores, dscores, g, st);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? ISOLOCO_OK : hip_fail(err, "gradient of routing");
}

}  // extern "C"
