// The embedding lookup and its gradient by sorted tokens.
//
//   out[t] = scale * table[id_t]
//   dtable[v] = scale * sum over t with id_t = v of dout[t]   (+ dtable[v])
//
// An id outside [0, vocab) holds no token: a row of zeros, and no gradient.
//
// Lookup: bounded by memory, every row read and written once.
//
// Gradient: the tokens are grouped by id first, then every row of the table is
// written once, from the sum of its tokens in the order they stand in (no
// atomics on the values: the same bits every time).  The grouping is one launch:
// workgroup b of NB owns the ids that are b modulo NB (frequent ids are
// neighbours in most vocabularies: this spreads them) and reads all ids, which
// come from the caches; it counts the tokens of workgroups before it, so no
// workgroup waits for another.  Ids with more than kPiece tokens are summed in
// pieces of the sorted order, which a last launch adds.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "isoloco_device.h"
#include "isoloco_error.h"

namespace isoloco {
namespace {

typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef floatx4 floatx4_any __attribute__((aligned(4)));

constexpr int kCols = 8;            // columns of a row that a lane holds
constexpr int kSpan = 64 * kCols;   // columns of a row that a wave holds

template <typename T>
__device__ __forceinline__ floatx8 load8(const T* p) {
  floatx8 r;
  if constexpr (sizeof(T) == 2) {
    const u32x4 v = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[2 * i] = bf16_to_f32(v[i] & 0xffffu);
      r[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  } else {
    const floatx4 a = *reinterpret_cast<const floatx4_any*>(p), b = *reinterpret_cast<const floatx4_any*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = a[i];
      r[4 + i] = b[i];
    }
  }
  return r;
}
// the first n of 8 values, zeros after them
template <typename T>
__device__ __forceinline__ floatx8 load8(const T* p, int n) {
  if (n >= kCols) return load8(p);
  floatx8 r;
#pragma unroll
  for (int i = 0; i < kCols; ++i) r[i] = i < n ? (float)p[i] : 0.f;
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, floatx8 v, int n) {
  if (n >= kCols) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4_any*>(p) = __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8_t));
    } else {
      *reinterpret_cast<floatx4_any*>(p) = (floatx4){v[0], v[1], v[2], v[3]};
      *reinterpret_cast<floatx4_any*>(p + 4) = (floatx4){v[4], v[5], v[6], v[7]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kCols; ++i)
    if (i < n) p[i] = (T)v[i];
}

// One wave per token and span of columns.
template <typename TT, typename TO, typename ID>
__global__ void __launch_bounds__(256) embed_kernel(const TT* table, int64_t ld_table, int64_t vocab, int dim,
                                                    const ID* ids, int64_t n, float scale, TO* out, int64_t ld_out,
                                                    int spans) {
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = item / spans;
  if (t >= n) return;
  const int col = (int)(item % spans) * kSpan + (threadIdx.x & 63) * kCols;
  if (col >= dim) return;
  const int64_t id = ids[t];
  const int left = dim - col;
  floatx8 v = {};
  if (id >= 0 && id < vocab) v = load8(table + id * ld_table + col, left) * scale;
  store8(out + t * ld_out + col, v, left);
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------

constexpr int kGroupThreads = 1024;
constexpr int kGroupWaves = kGroupThreads / 64;
constexpr int kMinGroups = 256;       // one workgroup per CU
constexpr int kGroupIds = 4096;       // most ids of a workgroup (16 KiB of LDS each for counts and cursors)
constexpr int kPiece = 64;            // tokens that one wave sums

// Workspace: the tokens grouped by id, the tokens as each workgroup found them,
// per id its first place and its count, the number of grouped tokens, and the
// sums of the pieces of frequent ids (two places per piece of the order: an id
// that ends in it and one that begins in it).
struct GroupTables {
  int32_t* order;   // n
  int32_t* found;   // n
  int32_t* first;   // vocab
  int32_t* count;   // vocab
  int32_t* total;   // 1
  float* piece;     // 2 * ceil(n / kPiece) * dim
};

int groups_of(int64_t vocab) {
  int nb = kMinGroups;
  while ((vocab + nb - 1) / nb > kGroupIds) nb *= 2;
  return nb;
}

template <typename ID>
__global__ void __launch_bounds__(kGroupThreads) group_kernel(const ID* ids, int32_t n, int64_t vocab, int nb_log2,
                                                             GroupTables g) {
  __shared__ int32_t cursor[kGroupIds];
  __shared__ int32_t wave_cnt[kGroupWaves], wave_before[kGroupWaves], wave_scan[kGroupWaves];
  const int nb = 1 << nb_log2, b = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = (int)((vocab - b + nb - 1) >> nb_log2);  // ids b, b + nb, ... below vocab
  for (int i = threadIdx.x; i < mine; i += kGroupThreads) cursor[i] = 0;
  __syncthreads();

  // each wave reads a run of tokens, twice: counts, then places
  const int run = ((n + kGroupWaves - 1) / kGroupWaves + 63) / 64 * 64;
  const int from = min((int64_t)n, (int64_t)wave * run), to = min((int64_t)n, (int64_t)from + run);
  int before = 0, cnt = 0;
  for (int t = from + lane; t < to; t += 64) {
    const int64_t id = ids[t];
    if (id >= 0 && id < vocab) {
      const int grp = (int)(id & (nb - 1));
      before += grp < b;
      if (grp == b) {
        ++cnt;
        atomicAdd(&cursor[id >> nb_log2], 1);
      }
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    before += __shfl_xor(before, off, 64);
    cnt += __shfl_xor(cnt, off, 64);
  }
  if (lane == 0) {
    wave_cnt[wave] = cnt;
    wave_before[wave] = before;
  }
  __syncthreads();
  int base = 0, at = 0, m = 0;
  for (int w = 0; w < kGroupWaves; ++w) {
    base += wave_before[w];
    if (w < wave) at += wave_cnt[w];
    m += wave_cnt[w];
  }
  if (b == nb - 1 && threadIdx.x == 0) *g.total = base + m;
  // the tokens of this workgroup in their order
  at += base;
  for (int t0 = from; t0 < to; t0 += 64) {
    const int t = t0 + lane;
    const int64_t id = t < to ? (int64_t)ids[t] : -1;
    const bool hit = id >= 0 && id < vocab && (int)(id & (nb - 1)) == b;
    const uint64_t mask = __ballot(hit);
    if (hit) g.found[at + __popcll(mask & ((1ull << lane) - 1))] = t;
    at += __popcll(mask);
  }
  // where each id's tokens go: its counts' running sum, 1024 ids a turn
  int carry = base;
  for (int i0 = 0; i0 < mine; i0 += kGroupThreads) {
    const int i = i0 + threadIdx.x;
    const int c = i < mine ? cursor[i] : 0;
    int s = c;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(s, off, 64);
      if (lane >= off) s += o;
    }
    __syncthreads();
    if (lane == 63) wave_scan[wave] = s;
    __syncthreads();
    int begin = carry + s - c;
    for (int w = 0; w < kGroupWaves; ++w) {
      if (w < wave) begin += wave_scan[w];
      carry += wave_scan[w];
    }
    if (i < mine) {
      cursor[i] = begin;
      const int64_t id = ((int64_t)i << nb_log2) + b;
      g.first[id] = begin;
      g.count[id] = c;
    }
  }
  __syncthreads();  // also: this workgroup's found[] is visible to all of it
  // each wave places the tokens of the ids that are its own modulo the waves
  for (int j0 = 0; j0 < m; j0 += 64) {
    const int j = j0 + lane;
    const int t = j < m ? g.found[base + j] : -1;
    const int local = t >= 0 ? (int)((int64_t)ids[t] >> nb_log2) : -1;
    uint64_t todo = __ballot(t >= 0 && (local & (kGroupWaves - 1)) == wave);
    while (todo) {
      const int lead = __ffsll((unsigned long long)todo) - 1;
      const int which = __shfl(local, lead, 64);
      const uint64_t same = __ballot(t >= 0 && local == which);
      int start = 0;
      if (lane == 0) {
        start = cursor[which];
        cursor[which] = start + __popcll(same);
      }
      start = __shfl(start, 0, 64);
      if ((same >> lane) & 1) g.order[start + __popcll(same & ((1ull << lane) - 1))] = t;
      todo &= ~same;
    }
  }
}

template <typename TD>
__device__ __forceinline__ floatx8 sum_tokens(const int32_t* order, int from, int to, const TD* dout, int64_t ld,
                                              int col, int left) {
  floatx8 s = {};
  for (int j = from; j < to; ++j) s += load8(dout + (int64_t)order[j] * ld + col, left);
  return s;
}

template <typename TG>
__device__ __forceinline__ void put_row(TG* dtable, int64_t at, floatx8 s, float scale, int accumulate, int left) {
  s *= scale;
  if (accumulate) s += load8(dtable + at, left);
  store8(dtable + at, s, left);
}

// Rows of at most kPiece tokens: one wave per id and span of columns.
template <typename TD, typename TG>
__global__ void __launch_bounds__(256) embed_rows_kernel(GroupTables g, const TD* dout, int64_t ld_dout, int64_t vocab,
                                                         int dim, float scale, int accumulate, TG* dtable,
                                                         int64_t ld_dtable, int spans) {
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t v = item / spans;
  if (v >= vocab) return;
  const int c = g.count[v];
  if (c > kPiece || (c == 0 && accumulate)) return;
  const int col = (int)(item % spans) * kSpan + (threadIdx.x & 63) * kCols;
  if (col >= dim) return;
  const int f = g.first[v];
  const floatx8 s = sum_tokens(g.order, f, f + c, dout, ld_dout, col, dim - col);
  put_row(dtable, v * ld_dtable + col, s, scale, accumulate, dim - col);
}

// The frequent ids that the piece [k kPiece, (k + 1) kPiece) of the order touches:
// such an id has more tokens than a piece, so it holds the piece's first or last place.
template <typename TD, typename ID>
__global__ void __launch_bounds__(256) embed_pieces_kernel(GroupTables g, const ID* ids, const TD* dout,
                                                           int64_t ld_dout, int dim, int spans, int pieces) {
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int k = (int)(item / spans);
  if (k >= pieces) return;
  const int col = (int)(item % spans) * kSpan + (threadIdx.x & 63) * kCols;
  const int total = *g.total, from = k * kPiece, to = min(total, from + kPiece);
  if (from >= to || col >= dim) return;
  const int64_t va = ids[g.order[from]], vb = ids[g.order[to - 1]];
  if (g.count[va] > kPiece)
    store8(g.piece + (int64_t)(2 * k) * dim + col,
           sum_tokens(g.order, from, min(to, g.first[va] + g.count[va]), dout, ld_dout, col, dim - col), dim - col);
  if (vb != va && g.count[vb] > kPiece)
    store8(g.piece + (int64_t)(2 * k + 1) * dim + col,
           sum_tokens(g.order, g.first[vb], to, dout, ld_dout, col, dim - col), dim - col);
}

// The frequent id that begins in a piece (at most one does), from its pieces' sums.
template <typename ID, typename TG>
__global__ void __launch_bounds__(64) embed_join_kernel(GroupTables g, const ID* ids, int dim, float scale,
                                                        int accumulate, TG* dtable, int64_t ld_dtable) {
  const int k = blockIdx.x, col = blockIdx.y * kSpan + threadIdx.x * kCols;
  const int total = *g.total, from = k * kPiece, to = min(total, from + kPiece);
  if (from >= to || col >= dim) return;
  const int64_t v = ids[g.order[to - 1]];
  const int f = g.first[v], c = g.count[v];
  if (c <= kPiece || f < from) return;
  const int left = dim - col;
  floatx8 s = load8(g.piece + (int64_t)(2 * k + (f > from)) * dim + col, left);
  for (int j = k + 1; j * kPiece < f + c; ++j) s += load8(g.piece + (int64_t)(2 * j) * dim + col, left);
  put_row(dtable, v * ld_dtable + col, s, scale, accumulate, left);
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Offsets of the tables in the workspace; returns its size.
size_t group_layout(int64_t n, int64_t vocab, int64_t dim, char* base, GroupTables* g) {
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    char* p = base + at;
    at += up256(bytes);
    return p;
  };
  GroupTables t;
  t.order = reinterpret_cast<int32_t*>(take(4 * (size_t)n));
  t.found = reinterpret_cast<int32_t*>(take(4 * (size_t)n));
  t.first = reinterpret_cast<int32_t*>(take(4 * (size_t)vocab));
  t.count = reinterpret_cast<int32_t*>(take(4 * (size_t)vocab));
  t.total = reinterpret_cast<int32_t*>(take(4));
  t.piece = reinterpret_cast<float*>(take(8 * (size_t)((n + kPiece - 1) / kPiece) * (size_t)dim));
  if (g) *g = t;
  return at;
}

isoloco_status check_table(int64_t vocab, int64_t dim, int64_t n, int32_t id_type) {
  if (vocab < 1 || vocab > kMaxExtent / 2 || dim < 1 || dim > kMaxExtent / 2 || n < 0 || n > kMaxExtent / 2)
    return fail(ISOLOCO_ERR_INVALID_ARG, "vocab %lld, dim %lld, %lld tokens", (long long)vocab, (long long)dim,
                (long long)n);
  if (!is_index_type(id_type)) return fail(ISOLOCO_ERR_INVALID_ARG, "id type %d", id_type);
  return ISOLOCO_OK;
}

// the blocks of a launch of `items` waves, four to a workgroup
bool wave_grid(int64_t items, unsigned* grid) {
  const int64_t blocks = (items + 3) / 4;
  *grid = (unsigned)blocks;
  return blocks <= INT32_MAX;
}

template <typename TD, typename TG, typename ID>
hipError_t run_backward(const GroupTables& g, const ID* ids, int64_t n, const TD* dout, int64_t ld_dout, int64_t vocab,
                        int dim, float scale, int accumulate, TG* dtable, int64_t ld_dtable, hipStream_t st) {
  const int spans = (dim + kSpan - 1) / kSpan, pieces = (int)((n + kPiece - 1) / kPiece);
  const int nb = groups_of(vocab);
  hipLaunchKernelGGL(group_kernel<ID>, dim3(nb), dim3(kGroupThreads), 0, st, ids, (int32_t)n, vocab,
                     __builtin_ctz(nb), g);
  unsigned grid;
  wave_grid(vocab * spans, &grid);
  hipLaunchKernelGGL((embed_rows_kernel<TD, TG>), dim3(grid), dim3(256), 0, st, g, dout, ld_dout, vocab, dim, scale,
                     accumulate, dtable, ld_dtable, spans);
  if (n > kPiece) {
    wave_grid((int64_t)pieces * spans, &grid);
    hipLaunchKernelGGL((embed_pieces_kernel<TD, ID>), dim3(grid), dim3(256), 0, st, g, ids, dout, ld_dout, dim, spans,
                       pieces);
    hipLaunchKernelGGL((embed_join_kernel<ID, TG>), dim3(pieces, spans), dim3(64), 0, st, g, ids, dim, scale,
                       accumulate, dtable, ld_dtable);
  }
  return hipGetLastError();
}

template <typename ID>
hipError_t pick_backward(const GroupTables& g, const void* ids, int64_t n, const void* dout, int64_t ld_dout,
                         int32_t dtype, int64_t vocab, int dim, float scale, int accumulate, void* dtable,
                         int64_t ld_dtable, int32_t dtable_dtype, hipStream_t st) {
  const ID* i = static_cast<const ID*>(ids);
  const float* df = static_cast<const float*>(dout);
  const __bf16* db = static_cast<const __bf16*>(dout);
  float* tf = static_cast<float*>(dtable);
  __bf16* tb = static_cast<__bf16*>(dtable);
  if (dtype == ISOLOCO_F32)
    return dtable_dtype == ISOLOCO_F32
               ? run_backward(g, i, n, df, ld_dout, vocab, dim, scale, accumulate, tf, ld_dtable, st)
               : run_backward(g, i, n, df, ld_dout, vocab, dim, scale, accumulate, tb, ld_dtable, st);
  return dtable_dtype == ISOLOCO_F32
             ? run_backward(g, i, n, db, ld_dout, vocab, dim, scale, accumulate, tf, ld_dtable, st)
             : run_backward(g, i, n, db, ld_dout, vocab, dim, scale, accumulate, tb, ld_dtable, st);
}

template <typename TT, typename TO, typename ID>
void run_lookup(const void* table, int64_t ld_table, int64_t vocab, int dim, const void* ids, int64_t n, float scale,
                void* out, int64_t ld_out, unsigned grid, int spans, hipStream_t st) {
  hipLaunchKernelGGL((embed_kernel<TT, TO, ID>), dim3(grid), dim3(256), 0, st, static_cast<const TT*>(table), ld_table,
                     vocab, dim, static_cast<const ID*>(ids), n, scale, static_cast<TO*>(out), ld_out, spans);
}

}  // namespace
}  // namespace isoloco

using namespace isoloco;

extern "C" {

isoloco_status isoloco_embedding(const void* table, int64_t ld_table, int32_t dtype, int64_t vocab, int64_t dim,
                                 const void* ids, int32_t id_type, int64_t n, float scale, void* out, int64_t ld_out,
                                 int32_t out_dtype, void* hip_stream) {
  ISOLOCO_TRY(check_table(vocab, dim, n, id_type));
  if (!is_dtype(dtype) || !is_dtype(out_dtype))
    return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d, out dtype %d", dtype, out_dtype);
  if (n == 0) return ISOLOCO_OK;
  const size_t et = dtype_bytes(dtype), eo = dtype_bytes(out_dtype), ei = index_bytes(id_type);
  ISOLOCO_TRY(check_matrix("table", table, vocab, dim, ld_table, et));
  ISOLOCO_TRY(check_matrix("out", out, n, dim, ld_out, eo));
  ISOLOCO_TRY(check_matrix("ids", ids, n, 1, 1, ei));
  const size_t ob = matrix_bytes(n, dim, ld_out, eo);
  if (ranges_overlap(out, ob, table, matrix_bytes(vocab, dim, ld_table, et)) ||
      ranges_overlap(out, ob, ids, (size_t)n * ei))
    return fail(ISOLOCO_ERR_ALIAS, "out overlaps the table or the ids");
  const int spans = (int)((dim + kSpan - 1) / kSpan);
  unsigned grid;
  if (!wave_grid(n * spans, &grid)) return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define LOOKUP(TT, TO, ID) \
  run_lookup<TT, TO, ID>(table, ld_table, vocab, (int)dim, ids, n, scale, out, ld_out, grid, spans, st)
  const bool tf = dtype == ISOLOCO_F32, of = out_dtype == ISOLOCO_F32;
  if (id_type == ISOLOCO_I32) {
    if (tf && of) LOOKUP(float, float, int32_t);
    else if (tf) LOOKUP(float, __bf16, int32_t);
    else if (of) LOOKUP(__bf16, float, int32_t);
    else LOOKUP(__bf16, __bf16, int32_t);
  } else {
    if (tf && of) LOOKUP(float, float, int64_t);
    else if (tf) LOOKUP(float, __bf16, int64_t);
    else if (of) LOOKUP(__bf16, float, int64_t);
    else LOOKUP(__bf16, __bf16, int64_t);
  }
#undef LOOKUP
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ISOLOCO_OK : hip_fail(e, "embedding");
}

isoloco_status isoloco_embedding_backward_workspace_size(int64_t n, int64_t vocab, int64_t dim, size_t* bytes) {
  if (!bytes) return fail(ISOLOCO_ERR_INVALID_ARG, "bytes is NULL");
  ISOLOCO_TRY(check_table(vocab, dim, n, ISOLOCO_I32));
  *bytes = group_layout(n, vocab, dim, nullptr, nullptr);
  return ISOLOCO_OK;
}

isoloco_status isoloco_embedding_backward(const void* ids, int32_t id_type, int64_t n, const void* dout,
                                          int64_t ld_dout, int32_t dtype, int64_t vocab, int64_t dim, float scale,
                                          int32_t accumulate, void* dtable, int64_t ld_dtable, int32_t dtable_dtype,
                                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  ISOLOCO_TRY(check_table(vocab, dim, n, id_type));
  if (!is_dtype(dtype) || !is_dtype(dtable_dtype))
    return fail(ISOLOCO_ERR_INVALID_ARG, "dtype %d, gradient's dtype %d", dtype, dtable_dtype);
  const size_t ed = dtype_bytes(dtype), et = dtype_bytes(dtable_dtype), ei = index_bytes(id_type);
  ISOLOCO_TRY(check_matrix("dout", dout, n, dim, ld_dout, ed));
  ISOLOCO_TRY(check_matrix("ids", ids, n, 1, 1, ei));
  ISOLOCO_TRY(check_matrix("dtable", dtable, vocab, dim, ld_dtable, et));
  GroupTables g;
  const size_t need = group_layout(n, vocab, dim, static_cast<char*>(workspace), &g);
  ISOLOCO_TRY(check_workspace(workspace, workspace_bytes, need));
  const size_t tb = matrix_bytes(vocab, dim, ld_dtable, et), db = matrix_bytes(n, dim, ld_dout, ed);
  if (ranges_overlap(dtable, tb, dout, db) || ranges_overlap(dtable, tb, ids, (size_t)n * ei) ||
      ranges_overlap(workspace, need, dtable, tb) || ranges_overlap(workspace, need, dout, db) ||
      ranges_overlap(workspace, need, ids, (size_t)n * ei))
    return fail(ISOLOCO_ERR_ALIAS, "dtable or the workspace overlaps another buffer");
  const int64_t spans = (dim + kSpan - 1) / kSpan;
  unsigned grid;
  if (!wave_grid(vocab * spans, &grid) || spans > 65535 || !wave_grid((n / kPiece + 1) * spans, &grid))
    return fail(ISOLOCO_ERR_UNSUPPORTED, "too many elements for one launch");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const hipError_t e =
      id_type == ISOLOCO_I32
          ? pick_backward<int32_t>(g, ids, n, dout, ld_dout, dtype, vocab, (int)dim, scale, accumulate, dtable,
                                   ld_dtable, dtable_dtype, st)
          : pick_backward<int64_t>(g, ids, n, dout, ld_dout, dtype, vocab, (int)dim, scale, accumulate, dtable,
                                   ld_dtable, dtable_dtype, st);
  return e == hipSuccess ? ISOLOCO_OK : hip_fail(e, "embedding gradient");
}

}  // extern "C"
