// The products grouped by expert on bfloat16 MFMA tiles (gfx950).
//
// Workgroups stay, one or two a CU, and go from tile to tile; slabs of 64 k values go from
// memory straight into LDS, one in flight while the one before is multiplied.  The products
// differ in how their operands lie:
//
//   kOut  rows of a (those that token names) against rows of the expert's matrix
//   kDx   rows of a against columns of the expert's matrix
//   kDw   columns of a against columns of b, over an expert's rows
//
// An expert's rows end inside tiles and slabs: what a load asks for past them it receives as
// zeros, by the bounds of its buffer.  Each XCD takes a run of the tiles, so that its L2 holds
// the operands that they share, cut by tiles (kDw: by their slabs, which differ from expert
// to expert).
//
// float32 operands are three bfloat16 parts each; their products are the same slabs six times
// over, one pair of parts after the other into the same accumulators, the smallest first.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_experts.h"
#include "isoloco_ffn.h"
#include "isoloco_slabs.h"

namespace isoloco {
namespace {

struct TileArgs {
  ExpertArgs g;
  int tiles_m, tiles_n, splits;  // tiles_m: of kDw
};

// A tile of the output, and its k values (kDw: rows of the operands).
struct Tile {
  int group, tm, tn, slice;
  int64_t begin, end;  // the group's rows
};

constexpr int kTileCost = 4;  // slabs that a tile's start and end take (bfloat16's: float32's are six times as long)

// The sum over the lanes up to this one
__device__ __forceinline__ int scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // a row of 16: 1, 2, 4, 8 lanes on
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last of a row to the next row
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the last of two rows to the other two
  return v;
}

// Lane `at`'s value, in scalar registers
__device__ __forceinline__ int64_t lane_of(int64_t v, int at) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, at), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), at);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Where the tiles lie, 64 experts at a time, one a lane: every wave by itself.  What an expert
// counts are its tiles, or (kDw, where all have as many) the slabs of its tiles (in 128s where
// the rows are many).  64 experts' counts fit 32 bits also where offsets fall and every expert
// has all rows: whatever they are, a tile lies inside the tensors.
template <ExpertProduct P, class C>
struct Finder {
  int64_t begin, end;  // of this lane's expert
  int own, upto;       // its count, and the counts up to it
  int base;            // of the 64
  __device__ __forceinline__ void load(const TileArgs& t, int first) {
    const int e = first + (threadIdx.x & 63);
    base = first;
    begin = end = 0;
    own = 0;
    if (e < t.g.groups.experts) {
      t.g.groups.rows_of(e, begin, end);
      const int many = t.g.groups.rows >> 24 ? 7 : 0;
      own = P == kDw ? (int)((end - begin + kSlab - 1) / kSlab >> many) + kTileCost * t.splits
                     : (int)((end - begin + C::TM - 1) / C::TM) * t.tiles_n * t.splits;
    }
    upto = scan(own);
  }
  // all counts
  __device__ __forceinline__ int64_t all(const TileArgs& t) {
    int64_t sum = 0;
    for (int first = 0; first < t.g.groups.experts; first += 64) {
      if (first != base) load(t, first);
      sum += __builtin_amdgcn_readlane(upto, 63);
    }
    return sum;
  }
  // the lane whose count passes `index`, and what is before the lane's 64; -1: none does
  __device__ __forceinline__ int pass(const TileArgs& t, int64_t index, int64_t& before) {
    before = 0;
    for (int first = 0; first < t.g.groups.experts; first += 64) {
      if (first != base) load(t, first);
      const uint64_t past = __ballot(before + upto > index);
      if (past) return __ffsll((unsigned long long)past) - 1;
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return -1;
  }
  // kDw: the tile that begins where the counts reach `index`
  __device__ __forceinline__ int64_t tile_at(const TileArgs& t, int64_t index) {
    const int64_t per = (int64_t)t.tiles_m * t.tiles_n * t.splits;
    int64_t before;
    const int at = pass(t, index, before);
    if (at < 0) return t.g.groups.experts * per;
    const int count = __builtin_amdgcn_readlane(own, at), past = __builtin_amdgcn_readlane(upto, at) - count;
    return (base + at) * per + (index - before - past) * per / count;
  }
  // The index-th tile.  Within an expert slices come first, then bands of 8 rows of tiles.
  __device__ __forceinline__ Tile tile(const TileArgs& t, int64_t index) {
    Tile o;
    int64_t i;
    if (P == kDw) {
      const int64_t per = (int64_t)t.tiles_m * t.tiles_n * t.splits;
      o.group = (int)(index / per);
      i = index - o.group * per;
      if (o.group < base || o.group >= base + 64) load(t, o.group & ~63);
      const int at = o.group - base;
      o.begin = lane_of(begin, at);
      o.end = lane_of(end, at);
    } else {
      int64_t before;
      const int at = pass(t, index, before);
      o.group = base + at;
      i = index - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(own, at));
      o.begin = lane_of(begin, at);
      o.end = lane_of(end, at);
    }
    const int tiles_m = P == kDw ? t.tiles_m : (int)((o.end - o.begin + C::TM - 1) / C::TM);
    const uint32_t plane = (uint32_t)tiles_m * t.tiles_n, band_of = 8u * t.tiles_n;
    o.slice = (int)((uint32_t)i / plane);
    uint32_t in = (uint32_t)i - o.slice * plane;
    const uint32_t band = in / band_of;
    in -= band * band_of;
    const uint32_t rows = min(8, tiles_m - (int)band * 8);
    o.tm = (int)(band * 8 + in % rows);
    o.tn = (int)(in / rows);
    return o;
  }
};

// Bytes from a place to the end of its buffer, as a buffer's size
__device__ __forceinline__ uint32_t bounded(int64_t bytes) { return (uint32_t)min(max(bytes, (int64_t)0), (int64_t)kMostBytes); }

template <class C>
struct TileLds {
  typedef Patch<C::NB * 32> P;
  static constexpr int kStage = (C::TM + C::TN) * 128, kWs = P::kBytes;
  static constexpr int kBytes = 2 * kStage > C::waves * kWs ? 2 * kStage : C::waves * kWs;
  static_assert(kBytes <= 160 * 1024, "LDS");
};

template <ExpertProduct P, bool F32, bool GATHER, class C>
__device__ __forceinline__ void multiply_tile(const TileArgs& t, const Tile& tile, char* lds) {
  constexpr bool ACOLS = P == kDw, BCOLS = P != kOut;
  typedef RowsSlab<C::TM, C::threads> AR;
  typedef ColsSlab<C::TM, C::threads> AC;
  typedef RowsSlab<C::TN, C::threads> BR;
  typedef ColsSlab<C::TN, C::threads> BC;
  constexpr int kA = C::TM * 128, kStage = TileLds<C>::kStage;
  typedef typename TileLds<C>::P Patch_;

  const ExpertArgs& g = t.g;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WN, wn = wave % C::WN;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int64_t len = tile.end - tile.begin, i0 = (int64_t)tile.tm * C::TM, j0 = (int64_t)tile.tn * C::TN;
  const int64_t m_all = P == kDw ? g.m : len;  // rows of this output
  const int64_t depth = P == kDw ? len : g.k;
  const int64_t row_a = 2 * g.ld_a, row_b = 2 * g.ld_b;  // bytes
  const int64_t gathered = 2 * g.tokens * (P == kDw ? g.ld_b : g.ld_a);  // bytes of what token reads

  AR ar;
  AC ac;
  BR br;
  BC bc;
  const char* a = reinterpret_cast<const char*>(g.a);
  const char* b = reinterpret_cast<const char*>(g.b);
  if constexpr (ACOLS) {
    a += tile.begin * row_a + 2 * i0;
    ac.init((uint32_t)row_a, g.cols_a - i0);
  } else if constexpr (GATHER) {
#pragma unroll
    for (int q = 0; q < AR::kLoads; ++q) {
      const int at = q * C::threads + threadIdx.x;
      const int64_t r = min((int64_t)(at >> 3), len - i0 - 1);
      const int64_t s = g.token.get(tile.begin + i0 + r);
      ar.vo[q] = s >= 0 && s < g.tokens ? (uint32_t)(s * row_a) + 16u * AR::piece(at) : kOutside;
    }
  } else {
    a += (tile.begin + i0) * row_a;
    ar.init((uint32_t)row_a, len - i0);
  }
  if constexpr (P == kOut) {
    b += 2 * (tile.group * g.stride_b) + j0 * row_b;
    br.init((uint32_t)row_b, g.n - j0);
  } else {
    if constexpr (P == kDx) b += 2 * (tile.group * g.stride_b + j0);
    else if constexpr (GATHER) b += 0;
    else b += tile.begin * row_b + 2 * j0;
    bc.init((uint32_t)row_b, g.cols_b - j0);
  }

  // the slabs of this workgroup: runs, one per pair of parts, of which a split takes some
  constexpr int kPairs = F32 ? 6 : 1;
  const int slabs = (int)((depth + kSlab - 1) / kSlab);
  const int64_t all = (int64_t)slabs * kPairs;
  const int64_t first = all * tile.slice / t.splits, total = all * (tile.slice + 1) / t.splits - first;
  int pair = slabs ? (int)(first / slabs) : 0, at_slab = (int)(first - (int64_t)pair * slabs);  // of the next slab to load

  // kDw, gathered: where the rows of b's next slab lie.  A wave loads pieces of kRows rows at a
  // time; one lane asks for a row's token a slab ahead and finds its place once that slab has
  // come, so that nothing waits for it, and the row's lanes take the place from that lane.  (Each
  // lane its own tokens: 1026 against 896 us for 131072 rows of 1408 against 2048 columns.)
  constexpr bool kSeek = P == kDw && GATHER;
  constexpr int kRows = 64 / BC::kPieces, kRowsAll = C::threads / BC::kPieces;
  const int lane_row = (lane / kRows % BC::kLoads) * kRowsAll + wave * kRows + lane % kRows;  // of a slab
  const uint32_t* tokens = static_cast<const uint32_t*>(g.token.p) + (g.token.wide ? 2 : 1) * tile.begin;
  const int last_row = (int)len - 1;
  uint32_t seek[BC::kLoads], token = 0, token_high = 0;
  const auto ask = [&]() {
    if constexpr (kSeek) {
      const int64_t r = min(at_slab * kSlab + lane_row, last_row);
      token = tokens[g.token.wide ? 2 * r : r];
      if (g.token.wide) token_high = tokens[2 * r + 1];
    }
  };
  const auto take = [&]() {
    if constexpr (kSeek) {
      const bool in = at_slab * kSlab + lane_row <= last_row && token_high == 0 && token < (uint32_t)g.tokens;
      const uint32_t place = in ? token * (uint32_t)row_b : kOutside;
#pragma unroll
      for (int q = 0; q < BC::kLoads; ++q) {
        // (16 bytes of the tile's columns: bc.vo less its row's; past kOutside they do not come round)
        const int k = q * kRowsAll + (int)threadIdx.x / BC::kPieces;
        seek[q] = __shfl(place, q * kRows + lane / BC::kPieces, 64) + (bc.vo[q] - (uint32_t)k * bc.row_bytes);
        asm volatile("" : "+v"(seek[q]));
      }
    }
  };

  // part 0: the next slab of a, part 1: that of b
  const auto issue = [&](int buf, int part) {
    const uint32_t at = lds0 + (uint32_t)buf * kStage;
    const int64_t s = at_slab, k_left = depth - s * kSlab;
    // the parts of a: 2 1 0 1 0 0, of b: 0 1 2 0 1 0
    const int64_t oa = F32 ? (0x046 >> (2 * pair) & 3) * g.part_a : 0, ob = F32 ? (0x124 >> (2 * pair) & 3) * g.part_b : 0;
    if (part == 0) {
      const uint64_t pa = (uint64_t)(a + 2 * oa);
      if constexpr (ACOLS) ac.load_bounded(at, pa + s * kSlab * row_a, bounded((k_left - 1) * row_a + 2 * (g.cols_a - i0)));
      else ar.load(at, pa + 128 * s, GATHER ? bounded(gathered - 128 * s) : kMostBytes, k_left);
      return;
    }
    const uint64_t pb = (uint64_t)(b + 2 * ob);
    if constexpr (P == kOut) {
      br.load(at + kA, pb + 128 * s, kMostBytes, k_left);
    } else if constexpr (kSeek) {
      const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const u32x4 r = tile_rsrc(pb + 2 * j0, bounded(gathered - 2 * j0));
#pragma unroll
      for (int q = 0; q < BC::kLoads; ++q) load_to_lds(at + kA + 16u * (q * C::threads + w * 64), r, seek[q], 0);
    } else {
      bc.load_bounded(at + kA, pb + s * kSlab * row_b, bounded((k_left - 1) * row_b + 2 * (g.cols_b - j0)));
    }
    if (++at_slab == slabs) {
      at_slab = 0;
      ++pair;
    }
  };

  floatx16 acc[C::NA][C::NB];
#pragma unroll
  for (int x = 0; x < C::NA; ++x)
#pragma unroll
    for (int y = 0; y < C::NB; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.f;

  struct Frags {
    bf16x8 a[C::NA], b[C::NB];
  };
  // the fragments of k values kk .. kk + 15 of the slab in buffer `buf`
  const auto read = [&](Frags& f, int buf, int kk) {
    const char* at = lds + buf * kStage;
    const char* bt = at + kA;
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      if constexpr (ACOLS) f.a[x] = AC::frag(at, (wm * C::NA + x) * 32, kk);
      else f.a[x] = AR::frag(at, (wm * C::NA + x) * 32, kk);
    }
#pragma unroll
    for (int y = 0; y < C::NB; ++y) {
      if constexpr (BCOLS) f.b[y] = BC::frag(bt, (wn * C::NB + y) * 32, kk);
      else f.b[y] = BR::frag(bt, (wn * C::NB + y) * 32, kk);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // The products of 16 k values (b first: a lane then holds 4 consecutive columns
  // of one row); a part of the next slab is asked for behind the first of them.
  const auto multiply = [&](const Frags& f, bool more, int buf, int part) {
#pragma unroll
    for (int x = 0; x < C::NA; ++x)
#pragma unroll
      for (int y = 0; y < C::NB; ++y) {
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[y], f.a[x], acc[x][y], 0, 0, 0);
        if (x == 0 && y == 1) {
          __builtin_amdgcn_sched_barrier(0);
          if (more) issue(buf, part);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    __builtin_amdgcn_sched_barrier(0);
  };

  // The fragments of 16 k values are read while those before are multiplied; once the last of
  // a slab are in registers its buffer is free, so that the wait for the next slab and the
  // first reads from it pass behind the last products of this one.
  if (total > 0) {
    ask();
    take();
    issue(0, 0);
    issue(0, 1);
    if (total > 1) ask();
    wait_slabs<0>();
    if (total > 1) take();
    Frags f[2];
    read(f[0], 0, 0);
    if (total > 1) issue(1, 0);
#pragma unroll 1
    for (int64_t s = 0; s < total; ++s) {
      const int buf = (int)(s & 1);
#pragma unroll
      for (int kk = 16; kk < kSlab; kk += 16) {
        read(f[(kk / 16) & 1], buf, kk);
        multiply(f[(kk / 16 + 1) & 1], kk == 16 && s + 1 < total, buf ^ 1, 1);
        if (kk == 16 && s + 2 < total) ask();
      }
      wait_slabs<0>();  // slab s + 1 is in LDS, and every wave is done reading slab s
      if (s + 2 < total) take();
      if (s + 1 < total) read(f[0], buf ^ 1, 0);
      multiply(f[1], s + 2 < total, buf, 0);
    }
  }
  __syncthreads();  // every wave is done with the operands: LDS is free

  // acc[x][y][4 q + e] = C(32 x + lane % 32, 32 y + 8 q + 4 (lane / 32) + e)
  const int64_t col0 = j0 + wn * C::NB * 32;
  const auto quad_of = [&](int x, int y, int q) {
    return (floatx4){acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
  };
  const int64_t row_base = P == kDw ? 0 : tile.begin;

  if (t.splits > 1) {
    // a split's sums (its columns are padded: a quad of them is inside or outside)
    const int64_t cols = ffn_pad(g.n), rows = P == kDw ? g.groups.experts * g.m : g.groups.rows;
    float* part = g.partial + (tile.slice * rows + (P == kDw ? tile.group * g.m : row_base)) * cols;
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      const int64_t row = i0 + (wm * C::NA + x) * 32 + (lane & 31);
      if (row >= m_all) continue;
#pragma unroll
      for (int y = 0; y < C::NB; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = col0 + 32 * y + 8 * q + 4 * (lane >> 5);
          if (col < cols) *reinterpret_cast<floatx4*>(part + row * cols + col) = quad_of(x, y, q);
        }
    }
    return;
  }

  const int64_t out_at = (P == kDw ? tile.group * g.stride_out : 0) + row_base * g.ld_out;
  if constexpr (F32) {
    float* out = static_cast<float*>(g.out) + out_at;
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      const int64_t row = i0 + (wm * C::NA + x) * 32 + (lane & 31);
      if (row >= m_all) continue;
#pragma unroll
      for (int y = 0; y < C::NB; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = col0 + 32 * y + 8 * q + 4 * (lane >> 5);
          if (col < g.n) store4(out + row * g.ld_out + col, quad_of(x, y, q), g.n - col);
        }
    }
  } else {
    char* ws = lds + wave * TileLds<C>::kWs;
    if (P == kDx && g.wide_out) {
      // half of the columns at a time (131072 rows of 2048 from 1408, 1074 MB: 835 us, 815 past the
      // caches; 911 with the quads going out as they are, 32 bytes of 32 rows at once)
      constexpr int kHalf = C::NB / 2, kLanes = kHalf * 8, kRows_ = 64 / kLanes;
      float* out = static_cast<float*>(g.out) + out_at;
#pragma unroll
      for (int x = 0; x < C::NA; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int y = 0; y < kHalf; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<floatx4*>(Patch_::quad(ws, 2 * (32 * y + 8 * q + 4 * (lane >> 5)))) =
                  quad_of(x, h * kHalf + y, q);
          wave_fence();
#pragma unroll
          for (int u = 0; u < 32 / kRows_; ++u) {
            const int r = u * kRows_ + lane / kLanes, c4 = lane % kLanes;
            const int64_t row = i0 + (wm * C::NA + x) * 32 + r, col = col0 + 32 * h * kHalf + 4 * c4;
            const floatx4 v = *reinterpret_cast<const floatx4*>(ws + r * Patch_::kPitch + c4 * 16);
            if (row >= m_all || col >= g.n) continue;
            float* to = out + row * g.ld_out + col;
            if (g.past && col + 4 <= g.n) __builtin_nontemporal_store(v, reinterpret_cast<floatx4_any*>(to));
            else store4(to, v, g.n - col);
          }
          wave_fence();
        }
      return;
    }
    uint16_t* out = static_cast<uint16_t*>(g.out) + out_at;
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
#pragma unroll
      for (int y = 0; y < C::NB; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<bf16x4*>(Patch_::quad(ws, 32 * y + 8 * q + 4 * (lane >> 5))) = rounded(quad_of(x, y, q));
      wave_fence();
      Patch_::store(ws, out, g.ld_out, i0 + (wm * C::NA + x) * 32, col0, m_all, g.n, m_all, g.n);
      wave_fence();
    }
  }
}

// The run of tiles [from, to) of a workgroup's XCD (workgroups go round the 8 XCDs in turn).
template <ExpertProduct P, class C>
__device__ __forceinline__ void run_of(const TileArgs& t, Finder<P, C>& finder, int64_t& from, int64_t& to) {
  const int xcd = blockIdx.x & 7;
  finder.load(t, 0);
  const int64_t all = finder.all(t);
  from = all * xcd / 8;
  to = all * (xcd + 1) / 8;
  if (P == kDw) {
    from = finder.tile_at(t, from);
    to = finder.tile_at(t, to);
  }
}

// Rows of no expert: zeros.
template <bool F32>
__device__ __forceinline__ void clear_rest(const ExpertArgs& g) {
  int64_t begin, end;
  g.groups.rows_of(g.groups.experts, begin, end);
  for (int64_t r = begin + blockIdx.x; r < end; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < g.n; c += blockDim.x) {
      if (F32 || g.wide_out) static_cast<float*>(g.out)[r * g.ld_out + c] = 0.f;
      else static_cast<uint16_t*>(g.out)[r * g.ld_out + c] = 0;
    }
}

template <ExpertProduct P, bool F32, bool GATHER, class C>
__global__ void __launch_bounds__(C::threads, 2) expert_tile_kernel(TileArgs t) {
  __shared__ __attribute__((aligned(1024))) char lds[TileLds<C>::kBytes];
  const int slot = blockIdx.x >> 3, slots = gridDim.x >> 3;
  Finder<P, C> finder;
  int64_t from, to;
  run_of(t, finder, from, to);
  for (int64_t i = from + slot; i < to; i += slots) {
    multiply_tile<P, F32, GATHER, C>(t, finder.tile(t, i), lds);
    __syncthreads();  // the results have left LDS
  }
  if (P != kDw && t.splits == 1) clear_rest<F32>(t.g);
}

// Both gradients: neither waits for the other, and where each alone has few tiles, or deep
// and shallow ones, they fill the card together.
template <bool F32, bool GATHER, class C>
__global__ void __launch_bounds__(C::threads, 2) expert_gradients_kernel(TileArgs w, TileArgs x) {
  __shared__ __attribute__((aligned(1024))) char lds[TileLds<C>::kBytes];
  const int slot = blockIdx.x >> 3, slots = gridDim.x >> 3;
  Finder<kDw, C> find_w;
  Finder<kDx, C> find_x;
  int64_t from_w, to_w, from_x, to_x;
  run_of(w, find_w, from_w, to_w);
  run_of(x, find_x, from_x, to_x);
  int64_t i = from_w + slot;
  for (; i < to_w; i += slots) {
    multiply_tile<kDw, F32, GATHER, C>(w, find_w.tile(w, i), lds);
    __syncthreads();
  }
  for (i += from_x - to_w; i < to_x; i += slots) {
    multiply_tile<kDx, F32, false, C>(x, find_x.tile(x, i), lds);
    __syncthreads();
  }
  if (x.splits == 1) clear_rest<F32>(x.g);
}

typedef bf16x4 bf16x4_any __attribute__((aligned(2)));

// The splits of a product added in their order.  One thread per quad of columns.
template <ExpertProduct P, bool F32>
__device__ __forceinline__ void join(const TileArgs& t, int64_t block) {
  const ExpertArgs& g = t.g;
  const int64_t cols = ffn_pad(g.n), rows = P == kDw ? g.groups.experts * g.m : g.groups.rows;
  const int64_t i = (block * 256 + threadIdx.x) * 4, row = i / cols, col = i - row * cols;
  if (row >= rows || col >= g.n) return;
  bool some = true;
  if (P != kDw) {
    int64_t begin, end;
    g.groups.rows_of(g.groups.experts, begin, end);
    some = row < begin;  // (rows of no expert: zeros)
  }
  floatx4 s = {};
  if (some)
    for (int k = 0; k < t.splits; ++k) s += *reinterpret_cast<const floatx4*>(g.partial + k * rows * cols + i);
  int64_t at = row * g.ld_out + col;
  if (P == kDw) {
    const int64_t e = row / g.m;
    at = e * g.stride_out + (row - e * g.m) * g.ld_out + col;
  }
  if (F32 || (P == kDx && g.wide_out)) {
    store4(static_cast<float*>(g.out) + at, s, g.n - col);
  } else {
    uint16_t* out = static_cast<uint16_t*>(g.out) + at;
    const bf16x4 r = rounded(s);
    if (col + 4 <= g.n) {
      *reinterpret_cast<bf16x4_any*>(out) = r;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < g.n) reinterpret_cast<__bf16*>(out)[e] = r[e];
    }
  }
}

template <ExpertProduct P, bool F32>
__global__ void __launch_bounds__(256) expert_join_kernel(TileArgs t) {
  join<P, F32>(t, blockIdx.x);
}

template <bool F32>
__global__ void __launch_bounds__(256) expert_join_gradients_kernel(TileArgs w, TileArgs x, int w_blocks) {
  const int block = blockIdx.x;
  if (block < w_blocks) join<kDw, F32>(w, block);
  else join<kDx, F32>(x, block - w_blocks);
}

// `most`: the most tiles that the experts' sizes can make.
template <ExpertProduct P, class C>
TileArgs tile_args(const ExpertArgs& g, int splits, int64_t& most) {
  TileArgs t;
  t.g = g;
  t.splits = splits;
  t.tiles_n = (int)((g.n + C::TN - 1) / C::TN);
  t.tiles_m = P == kDw ? (int)((g.m + C::TM - 1) / C::TM) : 0;
  const int64_t tiles_m = P == kDw ? (int64_t)g.groups.experts * t.tiles_m
                                   : g.groups.rows / C::TM + std::min<int64_t>(g.groups.rows, g.groups.experts);
  most = tiles_m * t.tiles_n * splits;
  return t;
}

template <ExpertProduct P>
unsigned join_blocks(const TileArgs& t) {
  const int64_t rows = P == kDw ? t.g.groups.experts * t.g.m : t.g.groups.rows;
  return t.splits > 1 ? (unsigned)((rows * ffn_pad(t.g.n) / 4 + 255) / 256) : 0;
}

// workgroups that stay: a multiple of 8, one for each XCD
template <class C>
unsigned stay(int64_t most) {
  return (unsigned)std::min<int64_t>((int64_t)kCus * (C::waves == 4 ? 2 : 1), (most + 7) / 8 * 8);
}

template <ExpertProduct P, bool F32, bool GATHER, class C>
hipError_t launch_shape(const ExpertArgs& g, int splits, hipStream_t st) {
  int64_t most;
  const TileArgs t = tile_args<P, C>(g, splits, most);
  hipLaunchKernelGGL((expert_tile_kernel<P, F32, GATHER, C>), dim3(stay<C>(most)), dim3(C::threads), 0, st, t);
  if (const unsigned b = join_blocks<P>(t))
    hipLaunchKernelGGL((expert_join_kernel<P, F32>), dim3(b), dim3(256), 0, st, t);
  return hipGetLastError();
}

template <ExpertProduct P, bool F32, bool GATHER>
hipError_t launch_gathered(const ExpertArgs& g, const ExpertPlan& p, hipStream_t st) {
  if (p.shape == kLarge) return launch_shape<P, F32, GATHER, Large>(g, p.splits, st);
  if constexpr (P != kDw) {
    if (p.shape == kMiddle) return launch_shape<P, F32, GATHER, Middle>(g, p.splits, st);
  }
  return launch_shape<P, F32, GATHER, Small>(g, p.splits, st);
}

template <ExpertProduct P, bool F32>
hipError_t launch_product(const ExpertArgs& g, const ExpertPlan& p, hipStream_t st) {
  if constexpr (P != kDx) {
    if (g.token.p) return launch_gathered<P, F32, true>(g, p, st);
  }
  return launch_gathered<P, F32, false>(g, p, st);
}

template <bool F32, bool GATHER, class C>
hipError_t launch_together(const ExpertArgs& dx, const ExpertArgs& dw, const ExpertGradients& p, hipStream_t st) {
  int64_t most_x, most_w;
  TileArgs x = tile_args<kDx, C>(dx, p.dx.splits, most_x), w = tile_args<kDw, C>(dw, p.dw.splits, most_w);
  x.g.partial += expert_partial_bytes(p.dw, kDw, dw.groups.rows, dw.groups.experts, dw.m, dw.n) / sizeof(float);
  hipLaunchKernelGGL((expert_gradients_kernel<F32, GATHER, C>), dim3(stay<C>(most_x + most_w)), dim3(C::threads), 0, st, w, x);
  const unsigned jw = join_blocks<kDw>(w), jx = join_blocks<kDx>(x);
  if (jw + jx) hipLaunchKernelGGL(expert_join_gradients_kernel<F32>, dim3(jw + jx), dim3(256), 0, st, w, x, (int)jw);
  return hipGetLastError();
}

// One of them alone goes by the same plan: the same bits.
template <bool F32>
hipError_t launch_gradients(const ExpertArgs* dx, const ExpertArgs* dw, hipStream_t st) {
  if (!dx && !dw) return hipSuccess;
  const ExpertArgs& any = dx ? *dx : *dw;
  const ExpertGradients p = expert_plan_gradients(F32, any.groups.rows, any.groups.experts, any.n, dx ? dx->k : dw->m);
  if (dx && dw && p.together) {
    const bool gather = dw->token.p;
    if (p.dw.shape == kLarge)
      return gather ? launch_together<F32, true, Large>(*dx, *dw, p, st) : launch_together<F32, false, Large>(*dx, *dw, p, st);
    return gather ? launch_together<F32, true, Small>(*dx, *dw, p, st) : launch_together<F32, false, Small>(*dx, *dw, p, st);
  }
  hipError_t e = hipSuccess;
  if (dx) e = launch_product<kDx, F32>(*dx, p.dx, st);
  if (e == hipSuccess && dw) e = launch_product<kDw, F32>(*dw, p.dw, st);
  return e;
}

}  // namespace

size_t expert_out_partial_bytes(bool f32, int64_t rows, int64_t experts, int64_t n, int64_t k) {
  return expert_partial_bytes(expert_plan(kOut, f32, rows, experts, 0, n, k), kOut, rows, experts, 0, n);
}

size_t expert_gradients_partial_bytes(bool f32, int64_t rows, int64_t experts, int64_t dim, int64_t cols) {
  const ExpertGradients p = expert_plan_gradients(f32, rows, experts, dim, cols);
  const size_t x = expert_partial_bytes(p.dx, kDx, rows, experts, 0, dim);
  const size_t w = expert_partial_bytes(p.dw, kDw, rows, experts, cols, dim);
  return p.together ? x + w : std::max(x, w);
}

hipError_t launch_expert_out(bool f32, const ExpertArgs& g, hipStream_t st) {
  const ExpertPlan p = expert_plan(kOut, f32, g.groups.rows, g.groups.experts, 0, g.n, g.k);
  return f32 ? launch_product<kOut, true>(g, p, st) : launch_product<kOut, false>(g, p, st);
}

hipError_t launch_expert_gradients(bool f32, const ExpertArgs* dx, const ExpertArgs* dw, hipStream_t st) {
  return f32 ? launch_gradients<true>(dx, dw, st) : launch_gradients<false>(dx, dw, st);
}

}  // namespace isoloco
