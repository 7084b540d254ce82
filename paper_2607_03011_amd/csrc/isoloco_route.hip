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
// No atomics decide an order: a workgroup counts its slots by expert, one launch adds the
// counts up over the workgroups, and each wave then places its slots in their order.
// Bounded by latency: the scores of 16384 tokens are a few MB; the choosing is top_k rounds
// of a maximum over a wave.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_error.h"
#include "isoloco_vec.h"

namespace isoloco {
namespace {

struct RouteArgs {
  int64_t ld, tokens;
  int experts, top_k, normalize;
  float* weight;
  int32_t *expert, *row, *token, *offsets;
  int32_t* counts;  // workgroups x (experts + 1); behind them the experts' totals
  int32_t* totals;
  int per_block;  // tokens of a workgroup
  int blocks;
};

constexpr int kSmallTokens = 64;     // so many are routed by one workgroup
constexpr int kSmallThreads = 1024;

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max64(v, (uint64_t)__shfl_xor((unsigned long long)v, off, 64));
  return v;
}

// One wave chooses a token's experts: lane j gets the j-th (-1: none), and its weight.
template <typename T, int EL>
__device__ __forceinline__ void choose(const T* scores, const RouteArgs& g, int& expert, float& weight) {
  const int lane = threadIdx.x & 63;
  uint64_t key[EL];
  float x[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = 64 * i + lane;
    x[i] = e < g.experts ? (float)scores[e] : -INFINITY;
    key[i] = e < g.experts ? key_of(x[i], (uint32_t)e) : 0;
  }
  uint64_t mine = 0;
  for (int j = 0; j < g.top_k; ++j) {
    uint64_t best = key[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) best = max64(best, key[i]);
    best = wave_max(best);
    if (lane == j) mine = best;
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (key[i] == best) key[i] = 0;
  }
  const float value = lane < g.top_k ? value_of(mine) : -INFINITY;
  const float m = __shfl(value, 0, 64);
  expert = value == -INFINITY ? -1 : (int)index_of(mine);
  float e = value == -INFINITY ? 0.f : expf(value - m), s = e;
  if (!g.normalize) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) s += x[i] == -INFINITY ? 0.f : expf(x[i] - m);
  }
  s = wave_sum(s);
  weight = expert < 0 ? 0.f : e / s;
}

// Where the experts' slots begin: the scan of `total` (experts + 1 groups) into `begin`, by one wave.
__device__ __forceinline__ void scan_groups(const int32_t* total, int groups, int32_t* begin) {
  const int lane = threadIdx.x & 63;
  int carry = 0;
  for (int base = 0; base < groups; base += 64) {
    const int i = base + lane, n = i < groups ? total[i] : 0;
    int sum = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(sum, off, 64);
      if (lane >= off) sum += o;
    }
    if (i < groups) begin[i] = carry + sum - n;
    carry += __shfl(sum, 63, 64);
  }
}

// One wave places the slots from `first` to `end` in their order; next[g] is the place of
// group g's next slot.  group_of(slot): its group.
template <typename GroupOf>
__device__ __forceinline__ void place(const RouteArgs& g, int64_t first, int64_t end, int32_t* next,
                                      const GroupOf& group_of) {
  const int lane = threadIdx.x & 63;
  int bits = 0;
  while ((1 << bits) <= g.experts) ++bits;  // groups are 0 .. experts
  for (int64_t base = first; base < end; base += 64) {
    const int64_t slot = base + lane;
    const bool live = slot < end;
    const int group = live ? group_of(slot) : 0;
    // the lanes of the same group
    uint64_t same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(group >> b & 1);
      same &= group >> b & 1 ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << lane) - 1));
    if (live) {
      const int at = next[group] + before;
      g.row[slot] = at;
      g.token[at] = (int32_t)(slot / g.top_k);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // (the group's last lane moves its place on)
    if (live && (same >> lane) == 1) next[group] += before + 1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Everything, by one workgroup.
template <typename T, int EL>
__global__ void __launch_bounds__(kSmallThreads) route_small_kernel(const T* scores, RouteArgs g) {
  __shared__ int32_t count[ISOLOCO_MAX_EXPERTS + 1], begin[ISOLOCO_MAX_EXPERTS + 1];
  __shared__ int16_t group[kSmallTokens * ISOLOCO_MAX_TOP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = g.experts + 1;
  for (int i = threadIdx.x; i < groups; i += kSmallThreads) count[i] = 0;
  __syncthreads();
  for (int t = wave; t < (int)g.tokens; t += kSmallThreads / 64) {
    int expert;
    float weight;
    choose<T, EL>(scores + t * g.ld, g, expert, weight);
    if (lane < g.top_k) {
      const int slot = t * g.top_k + lane;
      g.weight[slot] = weight;
      g.expert[slot] = expert;
      group[slot] = (int16_t)(expert < 0 ? g.experts : expert);
      atomicAdd(&count[group[slot]], 1);
    }
  }
  __syncthreads();
  if (wave > 0) return;
  scan_groups(count, groups, begin);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int i = lane; i < groups; i += 64) g.offsets[i] = begin[i];
  place(g, 0, g.tokens * g.top_k, begin, [&](int64_t slot) { return (int)group[slot]; });
}

// The choice of a workgroup's tokens, and its slots' counts by expert.
template <typename T, int EL>
__global__ void __launch_bounds__(256) route_choose_kernel(const T* scores, RouteArgs g) {
  __shared__ int32_t count[ISOLOCO_MAX_EXPERTS + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = g.experts + 1;
  for (int i = threadIdx.x; i < groups; i += 256) count[i] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * g.per_block, end = min(g.tokens, first + g.per_block);
  for (int64_t t = first + wave; t < end; t += 4) {
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
  for (int i = threadIdx.x; i < groups; i += 256) g.counts[(int64_t)blockIdx.x * groups + i] = count[i];
}

// The counts of the workgroups before each, and the totals: 64 groups per workgroup, its
// waves a run of the workgroups' counts each.
constexpr int kScanWaves = 16;
__global__ void __launch_bounds__(64 * kScanWaves) route_scan_kernel(RouteArgs g) {
  __shared__ int32_t sums[kScanWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = g.experts + 1;
  const int group = blockIdx.x * 64 + lane, per = (g.blocks + kScanWaves - 1) / kScanWaves;
  const int first = min(wave * per, g.blocks), end = min(first + per, g.blocks);
  const bool live = group < groups;
  int sum = 0;
  if (live)
    for (int b = first; b < end; ++b) sum += g.counts[(int64_t)b * groups + group];
  sums[wave][lane] = sum;
  __syncthreads();
  if (!live) return;
  int before = 0, total = 0;
  for (int w = 0; w < kScanWaves; ++w) {
    before += w < wave ? sums[w][lane] : 0;
    total += sums[w][lane];
  }
  for (int b = first; b < end; ++b) {
    int32_t* c = g.counts + (int64_t)b * groups + group;
    const int n = *c;
    *c = before;
    before += n;
  }
  if (wave == 0) g.totals[group] = total;
}

// One wave per workgroup of the choice.
__global__ void __launch_bounds__(64) route_place_kernel(RouteArgs g) {
  __shared__ int32_t next[ISOLOCO_MAX_EXPERTS + 1];
  const int lane = threadIdx.x, groups = g.experts + 1;
  scan_groups(g.totals, groups, next);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int i = lane; i < groups; i += 64) {
    if (blockIdx.x == 0) g.offsets[i] = next[i];
    next[i] += g.counts[(int64_t)blockIdx.x * groups + i];
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int64_t first = (int64_t)blockIdx.x * g.per_block, end = min(g.tokens, first + g.per_block);
  place(g, first * g.top_k, end * g.top_k, next, [&](int64_t slot) {
    const int e = g.expert[slot];
    return e < 0 ? g.experts : e;
  });
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
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
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
  s = wave_sum(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
  w *= inv;
  const float inner = wave_sum(w * grad);
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

// Tokens of a workgroup: 64, or more where that makes too many workgroups' counts.
int per_block_of(int64_t tokens) {
  int64_t n = 64;
  while ((tokens + n - 1) / n > 4096) n *= 2;
  return (int)n;
}

size_t route_workspace(int64_t tokens, int64_t experts) {
  if (tokens <= kSmallTokens) return 0;
  const int64_t per = per_block_of(tokens);
  return (size_t)((tokens + per - 1) / per + 1) * (size_t)(experts + 1) * 4;
}

template <typename T, int EL>
void run_forward(const void* scores, const RouteArgs& g, hipStream_t st) {
  const T* s = static_cast<const T*>(scores);
  if (g.tokens <= kSmallTokens) {
    hipLaunchKernelGGL((route_small_kernel<T, EL>), dim3(1), dim3(kSmallThreads), 0, st, s, g);
    return;
  }
  hipLaunchKernelGGL((route_choose_kernel<T, EL>), dim3(g.blocks), dim3(256), 0, st, s, g);
  hipLaunchKernelGGL(route_scan_kernel, dim3(g.experts / 64 + 1), dim3(64 * kScanWaves), 0, st, g);
  hipLaunchKernelGGL(route_place_kernel, dim3(g.blocks), dim3(64), 0, st, g);
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
  g.per_block = per_block_of(tokens);
  g.blocks = (int)((tokens + g.per_block - 1) / g.per_block);
  g.counts = static_cast<int32_t*>(workspace);
  g.totals = g.counts + (int64_t)g.blocks * (experts + 1);
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
