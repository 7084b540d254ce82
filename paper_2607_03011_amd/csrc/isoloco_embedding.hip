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
// come from the caches; it counts the tokens of the groups before its own, so no
// workgroup waits for another.  Ids with more than kPiece tokens are summed in
// pieces of the sorted order, which a last launch adds.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "isoloco_device.h"
#include "isoloco_error.h"

namespace isoloco {
namespace {

typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// N (4 or 8) columns of a row: as stored, and as float32.  A lane holds N, a wave 64 N.
template <int N>
struct Cols {
  typedef float F __attribute__((ext_vector_type(N)));
  template <typename T>
  struct Raw {
    static constexpr int kBytes = N * sizeof(T);
    uint32_t v[kBytes / 4];
    // the first n of them, zeros after those
    __device__ __forceinline__ void load(const T* p, int n) {
      if (n >= N) {
        if constexpr (kBytes == 8) {
          __builtin_memcpy(v, reinterpret_cast<const u32x2_any*>(p), 8);
        } else {
#pragma unroll
          for (int i = 0; i < kBytes / 16; ++i) {
            const u32x4 x = *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const char*>(p) + 16 * i);
            __builtin_memcpy(v + 4 * i, &x, 16);
          }
        }
      } else {
        T x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < n ? p[i] : (T)0.f;
        __builtin_memcpy(v, x, kBytes);
      }
    }
    __device__ __forceinline__ F get() const {
      F r;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 2) r[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
        else r[i] = __uint_as_float(v[i]);
      }
      return r;
    }
  };
  template <typename T>
  __device__ static __forceinline__ F load(const T* p, int n) {
    Raw<T> r;
    r.load(p, n);
    return r.get();
  }
  template <typename T>
  __device__ static __forceinline__ void store(T* p, F x, int n) {
    typedef T TN __attribute__((ext_vector_type(N)));
    const TN r = __builtin_convertvector(x, TN);
    if (n >= N) {
      if constexpr (N * sizeof(T) == 8) {
        *reinterpret_cast<u32x2_any*>(p) = __builtin_bit_cast(u32x2, r);
      } else {
        u32x4 w[N * sizeof(T) / 16];
        __builtin_memcpy(w, &r, sizeof w);
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i)
          *reinterpret_cast<u32x4_any*>(reinterpret_cast<char*>(p) + 16 * i) = w[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < n) p[i] = r[i];
    }
  }
};

// Columns per lane: 16 bytes of the rows that are written (lookup) or read (gradient), so
// that a wave's access is one run of memory.
template <typename T>
constexpr int kColsOf = 16 / sizeof(T);

// One wave per token and span of columns.
template <typename TT, typename TO, typename ID>
__global__ void __launch_bounds__(256) embed_kernel(const TT* table, int64_t ld_table, int64_t vocab, int dim,
                                                    const ID* ids, int64_t n, float scale, TO* out, int64_t ld_out,
                                                    int spans) {
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = item / spans;
  if (t >= n) return;
  typedef Cols<kColsOf<TO>> C;
  const int col = ((int)(item % spans) * 64 + (threadIdx.x & 63)) * kColsOf<TO>;
  if (col >= dim) return;
  const int64_t id = ids[t];
  const int left = dim - col;
  typename C::F v = {};
  if (id >= 0 && id < vocab) v = C::load(table + id * ld_table + col, left) * scale;
  C::store(out + t * ld_out + col, v, left);
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------

constexpr int kGroupThreads = 1024;
constexpr int kGroupWaves = kGroupThreads / 64;
constexpr int kMinGroups = 256;       // one workgroup per CU
constexpr int kGroupIds = 1024;       // most ids of a workgroup (a count per wave: 64 KiB of LDS)
constexpr int kPiece = 64;            // tokens that one wave sums

// Workspace: the tokens grouped by id, per id its first place and its count, the number of grouped tokens, and the
// sums of the pieces of frequent ids (two places per piece of the order: an id
// that ends in it and one that begins in it).
struct GroupTables {
  int32_t* order;   // n
  int2* row;        // vocab: an id's first place and its count
  int32_t* total;   // 1
  float* piece;     // 2 * ceil(n / kPiece) * dim
};

int groups_of(int64_t vocab) {
  int nb = kMinGroups;
  while ((vocab + nb - 1) / nb > kGroupIds) nb *= 2;
  return nb;
}

// Each wave takes a run of the tokens, a chunk at a time, kHeld per lane; a run of one chunk
// stays in registers between the counting and the placing.
template <typename ID, int kHeld>
__global__ void __launch_bounds__(kGroupThreads) group_kernel(const ID* ids, int32_t n, int64_t vocab, int nb_log2,
                                                             GroupTables g) {
  constexpr int kChunk = 64 * kHeld;
  // each wave's tokens by id; then where the next of them goes
  __shared__ int32_t cursor[kGroupWaves][kGroupIds];
  __shared__ int32_t wave_before[kGroupWaves], wave_scan[kGroupWaves];
  const int nb = 1 << nb_log2, b = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = (int)((vocab - b + nb - 1) >> nb_log2);  // ids b, b + nb, ... below vocab
  for (int i = lane; i < mine; i += 64) cursor[wave][i] = 0;

  const int run = ((n + kGroupWaves - 1) / kGroupWaves + 63) / 64 * 64;
  const int from = (int)min((int64_t)n, (int64_t)wave * run), to = (int)min((int64_t)n, (int64_t)from + run);
  // this lane's ids of the chunk from `at` on, -1 where there is no token, and per 64 of
  // them which are of this group
  int32_t held[kHeld];
  uint64_t mask[kHeld];
  const auto load = [&](int at) {
    constexpr int kAtOnce = kHeld < 16 ? kHeld : 16;
#pragma unroll
    for (int h = 0; h < kHeld; h += kAtOnce) {
      ID id[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        const int t0 = at + (h + q) * 64, t = t0 + lane;
        id[q] = (ID)-1;
        if (t0 < to && t < to) id[q] = ids[t];
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        bool valid = (uint32_t)id[q] < (uint32_t)vocab;  // (vocab is below 2^31)
        if constexpr (sizeof(ID) == 8) valid = valid && (uint32_t)((uint64_t)id[q] >> 32) == 0;
        held[h + q] = valid ? (int32_t)id[q] : -1;
        mask[h + q] = __ballot((held[h + q] & (int32_t)(0x80000000u | (nb - 1))) == b);
      }
    }
  };
  int before = 0;  // tokens of the groups before this one
  for (int at = from; at < to; at += kChunk) {
    load(at);
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
      before += (held[q] & (nb - 1)) < b;  // (-1 is in the last group here: before none)
      if (mask[q] && ((mask[q] >> lane) & 1)) atomicAdd(&cursor[wave][held[q] >> nb_log2], 1);
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off, 64);
  if (lane == 0) wave_before[wave] = before;
  __syncthreads();
  // where each id's tokens go: the running sum of the ids' counts, one id per thread, and
  // of the waves' in it
  const int i = threadIdx.x;
  int cnt[kGroupWaves], c = 0, base = 0;
#pragma unroll
  for (int w = 0; w < kGroupWaves; ++w) {
    cnt[w] = i < mine ? cursor[w][i] : 0;
    c += cnt[w];
    base += wave_before[w];
  }
  int s = c;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(s, off, 64);
    if (lane >= off) s += o;
  }
  if (lane == 63) wave_scan[wave] = s;
  __syncthreads();
  int begin = base + s - c, m = 0;
  for (int w = 0; w < kGroupWaves; ++w) {
    if (w < wave) begin += wave_scan[w];
    m += wave_scan[w];
  }
  if (i < mine) {
    g.row[((int64_t)i << nb_log2) + b] = make_int2(begin, c);
#pragma unroll
    for (int w = 0; w < kGroupWaves; ++w) {
      cursor[w][i] = begin;
      begin += cnt[w];
    }
  }
  if (b == nb - 1 && i == 0) *g.total = base + m;
  __syncthreads();
  for (int at = from; at < to; at += kChunk) {
    if (run > kChunk) load(at);
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
      uint64_t todo = mask[q];
      while (todo) {
        const int id = __builtin_amdgcn_readlane(held[q], __ffsll((unsigned long long)todo) - 1);
        const uint64_t same = __ballot(held[q] == id);
        int start = 0;
        if (lane == 0) {
          start = cursor[wave][id >> nb_log2];
          cursor[wave][id >> nb_log2] = start + __popcll(same);
        }
        start = __builtin_amdgcn_readfirstlane(start);
        if ((same >> lane) & 1) g.order[start + __popcll(same & ((1ull << lane) - 1))] = at + q * 64 + lane;
        todo &= ~same;
      }
    }
  }
}

// The sum of the c <= 64 tokens that the lanes hold (`t` of lane j is the j-th), with
// 32 registers' worth of rows in flight (64 leave room for five waves a SIMD instead of seven:
// 103 against 95 us for 32768 tokens of 2048).
template <int N, typename TD>
__device__ __forceinline__ typename Cols<N>::F sum_tokens(int t, int c, const TD* dout, int64_t ld, int col, int left) {
  typedef typename Cols<N>::template Raw<TD> Raw;
  typename Cols<N>::F s = {};
  int j = 0;
  const auto take = [&](auto ahead) {
    constexpr int kAhead = decltype(ahead)::value;
    Raw v[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) v[a].load(dout + (int64_t)__builtin_amdgcn_readlane(t, j + a) * ld + col, left);
#pragma unroll
    for (int a = 0; a < kAhead; ++a) s += v[a].get();
    j += kAhead;
  };
  constexpr int kMost = 128 / Raw::kBytes;
  while (j + kMost <= c) take(std::integral_constant<int, kMost>());
  while (j + 4 <= c) take(std::integral_constant<int, 4>());
  while (j < c) take(std::integral_constant<int, 1>());
  return s;
}

template <int N, typename TG>
__device__ __forceinline__ void put_row(TG* dtable, int64_t at, typename Cols<N>::F s, float scale, int accumulate,
                                        int left) {
  s *= scale;
  if (accumulate) s += Cols<N>::load(dtable + at, left);
  Cols<N>::store(dtable + at, s, left);
}

// The frequent ids that the piece [k kPiece, (k + 1) kPiece) of the order touches:
// such an id has more tokens than a piece, so it holds the piece's first or last place.
template <int N, typename TD, typename ID>
__device__ __forceinline__ void sum_piece(const GroupTables& g, const ID* ids, const TD* dout, int64_t ld_dout, int dim,
                                          int k, int col) {
  const int lane = threadIdx.x & 63;
  const int total = *g.total, from = k * kPiece, c = min(total - from, kPiece);
  if (c <= 0) return;
  const int t = g.order[from + min(lane, c - 1)];
  const int64_t va = ids[__builtin_amdgcn_readlane(t, 0)], vb = ids[__builtin_amdgcn_readlane(t, c - 1)];
  const int2 ra = g.row[va], rb = g.row[vb];
  if (ra.y > kPiece) {
    const auto s = sum_tokens<N>(t, min(c, ra.x + ra.y - from), dout, ld_dout, col, dim - col);
    if (col < dim) Cols<N>::store(g.piece + (int64_t)(2 * k) * dim + col, s, dim - col);
  }
  if (vb != va && rb.y > kPiece) {
    const int skip = rb.x - from;  // lane j then holds the j-th token of vb
    const auto s =
        sum_tokens<N>(__shfl(t, min(lane + skip, c - 1), 64), c - skip, dout, ld_dout, col, dim - col);
    if (col < dim) Cols<N>::store(g.piece + (int64_t)(2 * k + 1) * dim + col, s, dim - col);
  }
}

// One wave per item, many items per wave: first the pieces of frequent ids (the longest
// items), then the rows of at most kPiece tokens, each times the spans of columns.  A
// row's place, count and tokens are loaded while the rows before it are summed: most
// rows have few tokens or none and cost little but the wait for those.
template <typename TD, typename TG, typename ID>
__global__ void __launch_bounds__(256) embed_sums_kernel(GroupTables g, const ID* ids, const TD* dout, int64_t ld_dout,
                                                         int64_t vocab, int dim, float scale, int accumulate,
                                                         TG* dtable, int64_t ld_dtable, int spans, int pieces) {
  constexpr int N = kColsOf<TD>;
  const int lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)gridDim.x * 4, first = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t piece_items = (int64_t)pieces * spans;
  int64_t item = first;
  for (; item < piece_items; item += waves) {
    const int k = (int)(item / spans);
    sum_piece<N>(g, ids, dout, ld_dout, dim, k, ((int)(item - (int64_t)k * spans) * 64 + lane) * N);
  }
  // the row and span of an item, and of the wave's next one
  struct Place {
    int64_t v;
    int span;
  };
  const int64_t step_v = waves / spans;
  const int step_span = (int)(waves - step_v * spans);
  const auto after = [&](Place p) {
    p.v += step_v;
    p.span += step_span;
    if (p.span >= spans) {
      p.span -= spans;
      ++p.v;
    }
    return p;
  };
  const auto row_of = [&](Place p) { return p.v < vocab ? g.row[p.v] : make_int2(0, 0); };
  const auto tokens_of = [&](int2 r) { return r.y > 0 && r.y <= kPiece ? g.order[r.x + min(lane, r.y - 1)] : 0; };
  Place at;
  at.v = (item - piece_items) / spans;
  at.span = (int)(item - piece_items - at.v * spans);
  Place to = after(at);
  int2 r = row_of(at), r_next = row_of(to);
  int t = tokens_of(r);
  while (at.v < vocab) {
    const Place then = after(to);
    const int2 r_then = row_of(then);
    const int t_next = tokens_of(r_next);
    const int col = (at.span * 64 + lane) * N, c = __builtin_amdgcn_readfirstlane(r.y);
    if (c <= kPiece && !(c == 0 && accumulate) && col < dim) {
      const auto s = sum_tokens<N>(t, c, dout, ld_dout, col, dim - col);
      put_row<N>(dtable, at.v * ld_dtable + col, s, scale, accumulate, dim - col);
    }
    at = to;
    to = then;
    r = r_next;
    r_next = r_then;
    t = t_next;
  }
}

// The frequent id that begins in a piece (at most one does), from its pieces' sums.
template <typename ID, typename TG>
__global__ void __launch_bounds__(64) embed_join_kernel(GroupTables g, const ID* ids, int dim, float scale,
                                                        int accumulate, TG* dtable, int64_t ld_dtable) {
  constexpr int N = kColsOf<TG>;
  typedef Cols<N> C;
  const int k = blockIdx.x, col = (blockIdx.y * 64 + threadIdx.x) * N;
  const int total = *g.total, from = k * kPiece, to = min(total, from + kPiece);
  if (from >= to || col >= dim) return;
  const int64_t v = ids[g.order[to - 1]];
  const int f = g.row[v].x, c = g.row[v].y;
  if (c <= kPiece || f < from) return;
  const int left = dim - col;
  typename C::F s = C::load(g.piece + (int64_t)(2 * k + (f > from)) * dim + col, left);
#pragma unroll 8
  for (int j = k + 1; j <= (f + c - 1) / kPiece; ++j) s += C::load(g.piece + (int64_t)(2 * j) * dim + col, left);
  put_row<N>(dtable, v * ld_dtable + col, s, scale, accumulate, left);
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
  t.row = reinterpret_cast<int2*>(take(8 * (size_t)vocab));
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
  return launchable(blocks, 256);
}

template <typename TD, typename TG, typename ID>
hipError_t run_backward(const GroupTables& g, const ID* ids, int64_t n, const TD* dout, int64_t ld_dout, int64_t vocab,
                        int dim, float scale, int accumulate, TG* dtable, int64_t ld_dtable, hipStream_t st) {
  constexpr int kSpan = 64 * kColsOf<TD>;
  const int spans = (dim + kSpan - 1) / kSpan, pieces = (int)((n + kPiece - 1) / kPiece);
  const int nb = groups_of(vocab);
  // (few tokens: without the turns that would find none.  Us a call with 8 / 32 ids a lane: 5001
  // tokens 26.0 / 29.4, 8192 91 / 94, 32768 126 / 124)
  if (n <= kGroupWaves * 64 * 8)
    hipLaunchKernelGGL((group_kernel<ID, 8>), dim3(nb), dim3(kGroupThreads), 0, st, ids, (int32_t)n, vocab,
                       __builtin_ctz(nb), g);
  else
    hipLaunchKernelGGL((group_kernel<ID, 32>), dim3(nb), dim3(kGroupThreads), 0, st, ids, (int32_t)n, vocab,
                       __builtin_ctz(nb), g);
  const int pieced = n > kPiece ? pieces : 0;
  // 7 workgroups of 4 waves are on a CU at a time; four times as many even out what the rows
  // cost (us a call at 1 / 2 / 4 / 8 / 16 times: 134 / 127 / 124 / 121 / 122 for 32768 tokens
  // of 2048 in bfloat16, 54 / 51 / 50 / 51 / 55 for 768 in float32, 30.1 / 27.5 / 26.0 / 28.4 /
  // 33.0 for 5001 of 612)
  const int64_t items = (vocab + pieced) * spans, blocks = std::min<int64_t>((items + 3) / 4, 4 * 7 * 256);
  hipLaunchKernelGGL((embed_sums_kernel<TD, TG, ID>), dim3((unsigned)blocks), dim3(256), 0, st, g, ids, dout, ld_dout,
                     vocab, dim, scale, accumulate, dtable, ld_dtable, spans, pieced);
  if (pieced)
    hipLaunchKernelGGL((embed_join_kernel<ID, TG>),
                       dim3(pieces, (dim + 64 * kColsOf<TG> - 1) / (64 * kColsOf<TG>)), dim3(64), 0, st, g, ids, dim,
                       scale, accumulate, dtable, ld_dtable);
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
  const int64_t span = 64 * (16 / (int64_t)eo);
  const int spans = (int)((dim + span - 1) / span);
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
  if (dim > 65535 * 256)
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
