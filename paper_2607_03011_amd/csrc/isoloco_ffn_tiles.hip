// The products of the gated feed-forward block on bfloat16 MFMA tiles (gfx950).
//
// One workgroup per output tile; slabs of 64 k values go from memory straight into
// LDS, one in flight while the one before is multiplied.  The products differ in
// how their operands lie (k along the rows or across them) and in what becomes of
// the accumulators, which never leave the registers before that:
//
//   kForward, kInner  x rows against rows of both weights, half a tile's columns
//                     each, so that g and u of one output are in one lane
//   kSum              da and du rows against columns of the weights, one after the
//                     other into the same accumulators
//   kPair             columns of da or du against columns of x
//
// float32 operands are three bfloat16 parts each; their products are the same slabs
// six times over, one pair of parts after the other into the same accumulators, the
// smallest first.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>

#include "isoloco_device.h"
#include "isoloco_ffn.h"
#include "isoloco_ffn_plan.h"
#include "isoloco_slabs.h"

namespace isoloco {
namespace {

// v = act(gate) up, or (kInner) v = dh up act'(gate) and w = dh act(gate)
template <int MODE, int ACT, bool F32>
__device__ __forceinline__ void gated(floatx4 gate, floatx4 up, floatx4 dh, floatx4& v, floatx4& w) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float f, df;
    activate<ACT, F32>(gate[e], f, df);
    v[e] = MODE == kInner ? dh[e] * up[e] * df : f * up[e];
    w[e] = dh[e] * f;
  }
}

// A quad of da and du, in parts if float32; zeros in the padding (whose columns are
// the last one's again in the accumulators, whose rows may hold anything).
template <bool F32>
__device__ __forceinline__ void store_inner(const FfnArgs& g, int64_t row, int64_t col, floatx4 v, floatx4 w) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (row >= g.m || col + e >= g.n) v[e] = w[e] = 0.f;
#pragma unroll
  for (int p = 0; p < (F32 ? kFfnParts : 1); ++p) {
    const int64_t at = p * g.part_out + row * g.ld_out + col;
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(g.out[0]) + at) = next_part(v);
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(g.out[1]) + at) = next_part(w);
  }
}

// Columns of a split's sums
__host__ __device__ inline int64_t partial_cols(int mode, const FfnArgs& g) {
  return mode == kForward || mode == kInner ? ffn_pad(g.n) : g.cols_b;
}

struct TileArgs {
  FfnArgs g;
  int tiles_m, tiles_n, planes, splits, tiles;  // tiles: of every plane and split
};

// The tile of a workgroup: workgroups go round the 8 XCDs in turn, so each XCD takes
// a run of tiles, in bands of 8 rows of tiles, whose operands its L2 then holds.
__device__ __forceinline__ void tile_of(const TileArgs& t, int block, int& tm, int& tn, int& z, int& slice) {
  const int xcd = block & 7, q = t.tiles >> 3, r = t.tiles & 7;
  int i = xcd * q + min(xcd, r) + (block >> 3);
  const int plane = t.tiles_m * t.tiles_n;
  slice = i / (plane * t.planes);
  i -= slice * plane * t.planes;
  z = i / plane;
  i -= z * plane;
  const int band = i / (8 * t.tiles_n), in = i - band * 8 * t.tiles_n;
  const int rows = min(8, t.tiles_m - band * 8);
  tm = band * 8 + in % rows;
  tn = in / rows;
}

// Bytes of LDS: two stages of slabs; afterwards the waves' results on their way out.
template <int MODE, class C>
struct TileLds {
  static constexpr bool DUAL = MODE == kForward || MODE == kInner;
  typedef Patch<(DUAL ? C::NB / 2 : C::NB) * 32> P;
  static constexpr int kStage = (C::TM + C::TN) * 128, kWs = (MODE == kInner ? 2 : 1) * P::kBytes;
  static constexpr int kBytes = 2 * kStage > C::waves * kWs ? 2 * kStage : C::waves * kWs;
  static_assert(kBytes <= 160 * 1024, "LDS");
};

// One workgroup's tile, workgroup `block` of a product's.
template <int MODE, int ACT, bool F32, class C>
__device__ __forceinline__ void multiply_tile(const TileArgs& t, int block, char* lds) {
  constexpr bool DUAL = MODE == kForward || MODE == kInner, ACOLS = MODE == kPair;
  constexpr int kCols = DUAL ? C::TN / 2 : C::TN;  // output columns of a tile
  typedef RowsSlab<C::TM, C::threads> AR;
  typedef ColsSlab<C::TM, C::threads> AC;
  typedef RowsSlab<C::TN / 2, C::threads> BR;
  typedef ColsSlab<C::TN, C::threads> BC;
  constexpr int kA = C::TM * 128, kStage = TileLds<MODE, C>::kStage, kWs = TileLds<MODE, C>::kWs;
  typedef typename TileLds<MODE, C>::P P;

  const FfnArgs& g = t.g;
  int tm, tn, z, slice;
  tile_of(t, block, tm, tn, z, slice);
  const int64_t i0 = (int64_t)tm * C::TM, j0 = (int64_t)tn * kCols;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WN, wn = wave % C::WN;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;

  AR ar;
  AC ac;
  BR br;
  BC bc;
  const uint16_t *a[2], *b[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    a[p] = g.a[MODE == kPair ? z : MODE == kSum ? p : 0] + i0 * (ACOLS ? 1 : g.ld_a);
    b[p] = g.b[MODE == kPair ? 0 : p] + j0 * (DUAL ? g.ld_b : 1);
  }
  if constexpr (ACOLS) ac.init(2u * (uint32_t)g.ld_a, ffn_pad(g.m) - i0);
  else ar.init(2u * (uint32_t)g.ld_a, g.m - i0);
  if constexpr (DUAL) br.init(2u * (uint32_t)g.ld_b, g.n - j0);
  else bc.init(2u * (uint32_t)g.ld_b, g.cols_b - j0);

  // A workgroup's slabs: runs of `slabs`, one per term (kSum) and pair of parts
  // (float32), one after the other; a split product's workgroup takes some of them.
  constexpr int kPairs = F32 ? 6 : 1, kRuns = (MODE == kSum ? 2 : 1) * kPairs;
  const int slabs = (int)((g.k + kSlab - 1) / kSlab);
  const int64_t all = (int64_t)slabs * kRuns;
  const int64_t first = all * slice / t.splits, total = all * (slice + 1) / t.splits - first;
  int run = slabs ? (int)(first / slabs) : 0, at_slab = (int)(first - (int64_t)run * slabs);  // of the next slab to load

  // part 0: the next slab of a, part 1: that of b
  const auto issue = [&](int buf, int part) {
    const uint32_t at = lds0 + (uint32_t)buf * kStage;
    const int s = at_slab, term = MODE == kSum ? run / kPairs : 0, pair = F32 ? run - term * kPairs : 0;
    // the parts of a: 2 1 0 1 0 0, of b: 0 1 2 0 1 0
    const int64_t oa = F32 ? (0x046 >> (2 * pair) & 3) * g.part_a : 0, ob = F32 ? (0x124 >> (2 * pair) & 3) * g.part_b : 0;
    if constexpr (DUAL) {
      const int64_t k_left = g.k - (int64_t)s * kSlab;
      if (k_left < kSlab) {
        char* to = lds + buf * kStage;
        if (part == 0) {
          ar.load_end(to, a[0] + oa, s, (int)k_left);
        } else {
          br.load_end(to + kA, b[0] + ob, s, (int)k_left);
          br.load_end(to + kA + BR::kBytes, b[1] + ob, s, (int)k_left);
        }
      } else if (part == 0) {
        ar.load(at, a[0] + oa, s);
      } else {
        br.load(at + kA, b[0] + ob, s);
        br.load(at + kA + BR::kBytes, b[1] + ob, s);
      }
    } else {
      if (part == 1) bc.load(at + kA, (term ? b[1] : b[0]) + ob, s, g.k - (int64_t)s * kSlab);
      else if constexpr (ACOLS) ac.load(at, a[0] + oa, s, kSlab);
      else ar.load(at, (term ? a[1] : a[0]) + oa, s);
    }
    if (part == 1 && ++at_slab == slabs) {
      at_slab = 0;
      ++run;
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
      if constexpr (DUAL)  // the first half of a wave's blocks is the gate's, the second the up projection's
        f.b[y] = BR::frag(bt, (y / (C::NB / 2)) * (C::TN / 2) + (wn * (C::NB / 2) + y % (C::NB / 2)) * 32, kk);
      else
        f.b[y] = BC::frag(bt, (wn * C::NB + y) * 32, kk);
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

  // The fragments of 16 k values are read while those before are multiplied; once
  // the last of a slab are in registers its buffer is free, so that the wait for
  // the next slab and the first reads from it pass behind the last products of this
  // one.  A slab's loads are issued in two parts behind products: 64 of them at
  // once keep the CU's address unit busy for about half a slab's time, in which
  // their waves would multiply nothing (all at the barrier: 639 us for the sum over
  // 2 x 5632 of 16384 x 2048 outputs, in two parts 611).
  if (total > 0) {
    issue(0, 0);
    issue(0, 1);
    wait_slabs<0>();
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
      }
      wait_slabs<0>();  // slab s + 1 is in LDS, and every wave is done reading slab s
      if (s + 1 < total) read(f[0], buf ^ 1, 0);
      multiply(f[1], s + 2 < total, buf, 0);
    }
  }
  __syncthreads();  // every wave is done with the operands: LDS is free

  // acc[x][y][4 q + e] = C(32 x + lane % 32, 32 y + 8 q + 4 (lane / 32) + e)
  constexpr int kOut = DUAL ? C::NB / 2 : C::NB;
  const int64_t col0 = j0 + wn * kOut * 32;
  const auto quad_of = [&](int x, int y, int q) {
    return (floatx4){acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
  };
  const auto inner = [&](int x, int y, int q, floatx4 dh, floatx4& v, floatx4& w) {
    gated<MODE, ACT, F32>(quad_of(x, y, q), quad_of(x, kOut + y, q), dh, v, w);
  };

  if (t.splits > 1) {
    // a split's sums (cols is a multiple of 8: a quad of columns is inside or outside)
    const int64_t cols = partial_cols(MODE, g), plane = g.m * cols;
    float* part = g.partial + (DUAL ? 2 * slice : slice * t.planes + z) * plane;
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      const int64_t row = i0 + (wm * C::NA + x) * 32 + (lane & 31);
      if (row >= g.m) continue;
#pragma unroll
      for (int y = 0; y < kOut; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = col0 + 32 * y + 8 * q + 4 * (lane >> 5);
          if (col >= cols) continue;
          float* o = part + row * cols + col;
          *reinterpret_cast<floatx4*>(o) = quad_of(x, y, q);
          if constexpr (DUAL) *reinterpret_cast<floatx4*>(o + plane) = quad_of(x, kOut + y, q);
        }
    }
    return;
  }

  if constexpr (F32) {
    const int64_t rows_pad = ffn_pad(g.m), cols_pad = ffn_pad(g.n);
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      const int64_t row = i0 + (wm * C::NA + x) * 32 + (lane & 31);
      if (row >= (MODE == kInner ? rows_pad : g.m)) continue;
#pragma unroll
      for (int y = 0; y < kOut; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = col0 + 32 * y + 8 * q + 4 * (lane >> 5);
          if constexpr (MODE == kInner) {
            if (col >= cols_pad) continue;
            floatx4 v = {}, w = {};
            if (row < g.m) inner(x, y, q, load4(static_cast<const float*>(g.dh) + row * g.ld_dh + col, g.n - col), v, w);
            store_inner<true>(g, row, col, v, w);
          } else {
            if (col >= g.n) continue;
            floatx4 v = quad_of(x, y, q), w;
            if constexpr (DUAL) inner(x, y, q, (floatx4){}, v, w);
            store4(static_cast<float*>(g.out[z]) + row * g.ld_out + col, v, g.n - col);
          }
        }
    }
  } else {
    char* ws = lds + wave * kWs;
    const int64_t rows_pad = MODE == kInner ? ffn_pad(g.m) : g.m, cols_pad = MODE == kInner ? ffn_pad(g.n) : g.n;
    uint16_t* out = static_cast<uint16_t*>(g.out[z]);
    P dh_of[MODE == kInner ? C::NA : 1];  // all of the wave's dh at once: one wait
    if constexpr (MODE == kInner) {
#pragma unroll
      for (int x = 0; x < C::NA; ++x)
        dh_of[x].fetch(static_cast<const uint16_t*>(g.dh), g.ld_dh, i0 + (wm * C::NA + x) * 32, col0, g.m, g.n);
    }
#pragma unroll
    for (int x = 0; x < C::NA; ++x) {
      const int64_t row0 = i0 + (wm * C::NA + x) * 32;
      if constexpr (MODE == kInner) {
        dh_of[x].put(ws);
        wave_fence();
      }
#pragma unroll
      for (int y = 0; y < kOut; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          char* at = P::quad(ws, 32 * y + 8 * q + 4 * (lane >> 5));
          floatx4 v = quad_of(x, y, q), w, dh = {};
          if constexpr (MODE == kInner) dh = __builtin_convertvector(*reinterpret_cast<const bf16x4*>(at), floatx4);
          if constexpr (DUAL) inner(x, y, q, dh, v, w);
          if constexpr (MODE == kInner) *reinterpret_cast<bf16x4*>(at + P::kBytes) = rounded(w);
          *reinterpret_cast<bf16x4*>(at) = rounded(v);
        }
      wave_fence();
      P::store(ws, out, g.ld_out, row0, col0, g.m, g.n, rows_pad, cols_pad);
      if constexpr (MODE == kInner)
        P::store(ws + P::kBytes, static_cast<uint16_t*>(g.out[1]), g.ld_out, row0, col0, g.m, g.n, rows_pad, cols_pad);
      wave_fence();
    }
  }
}

template <int MODE, int ACT, bool F32, class C>
__global__ void __launch_bounds__(C::threads, 2) ffn_tile_kernel(TileArgs t) {
  __shared__ __attribute__((aligned(1024))) char lds[TileLds<MODE, C>::kBytes];
  multiply_tile<MODE, ACT, F32, C>(t, blockIdx.x, lds);
}

// Both products of the gradients in one launch: neither waits for the other, and where
// each alone has few tiles they fill the card together.
template <bool F32, class CS, class CP>
__global__ void __launch_bounds__(CS::threads, 2) ffn_gradients_kernel(TileArgs sum, TileArgs pair) {
  static_assert(CS::threads == CP::threads, "one launch");
  constexpr int kS = TileLds<kSum, CS>::kBytes, kP = TileLds<kPair, CP>::kBytes;
  __shared__ __attribute__((aligned(1024))) char lds[kS > kP ? kS : kP];
  const int block = blockIdx.x;
  if (block < sum.tiles) multiply_tile<kSum, ISOLOCO_ACT_SILU, F32, CS>(sum, block, lds);
  else multiply_tile<kPair, ISOLOCO_ACT_SILU, F32, CP>(pair, block - sum.tiles, lds);
}

typedef bf16x4 bf16x4_any __attribute__((aligned(2)));

template <bool F32>
__device__ __forceinline__ void store_out(void* out, floatx4 v, int64_t left) {
  if constexpr (F32) {
    store4(static_cast<float*>(out), v, left);
  } else {
    const bf16x4 r = rounded(v);
    if (left >= 4) {
      *static_cast<bf16x4_any*>(out) = r;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) static_cast<__bf16*>(out)[e] = r[e];
    }
  }
}

// The splits of a product added in their order, and what the tiles would have made of
// the whole sums.  One thread per quad of columns.
template <int MODE, int ACT, bool F32>
__device__ __forceinline__ void join(const TileArgs& t, int64_t block) {
  constexpr bool DUAL = MODE == kForward || MODE == kInner;
  const FfnArgs& g = t.g;
  const int64_t cols = partial_cols(MODE, g), plane = g.m * cols;
  const int64_t quads = (MODE == kInner ? ffn_pad(g.m) : g.m) * cols / 4;
  const int64_t at = block * 256 + threadIdx.x;
  const int z = MODE == kPair ? (int)(at / quads) : 0;
  const int64_t i = (at - z * quads) * 4, row = i / cols, col = i - row * cols;
  if (at >= quads * t.planes) return;
  const auto sum = [&](const float* p, int64_t step) {
    floatx4 s = *reinterpret_cast<const floatx4*>(p);
    for (int k = 1; k < t.splits; ++k) s += *reinterpret_cast<const floatx4*>(p + k * step);
    return s;
  };
  const int64_t size = F32 ? 4 : 2;
  if constexpr (DUAL) {
    floatx4 v = {}, w = {}, dh = {};
    if (row < g.m) {
      if constexpr (MODE == kInner) {
        if constexpr (F32) {
          dh = load4(static_cast<const float*>(g.dh) + row * g.ld_dh + col, g.n - col);
        } else {
          const __bf16* p = static_cast<const __bf16*>(g.dh) + row * g.ld_dh + col;
#pragma unroll
          for (int e = 0; e < 4; ++e) dh[e] = col + e < g.n ? (float)p[e] : 0.f;
        }
      }
      gated<MODE, ACT, F32>(sum(g.partial + i, 2 * plane), sum(g.partial + plane + i, 2 * plane), dh, v, w);
    }
    if constexpr (MODE == kInner) store_inner<F32>(g, row, col, v, w);
    else if (col < g.n) store_out<F32>(static_cast<char*>(g.out[0]) + (row * g.ld_out + col) * size, v, g.n - col);
  } else {
    if (col < g.n)
      store_out<F32>(static_cast<char*>(g.out[z]) + (row * g.ld_out + col) * size,
                     sum(g.partial + z * plane + i, t.planes * plane), g.n - col);
  }
}

template <int MODE, int ACT, bool F32>
__global__ void __launch_bounds__(256) ffn_join_kernel(TileArgs t) {
  join<MODE, ACT, F32>(t, blockIdx.x);
}

template <bool F32>
__global__ void __launch_bounds__(256) ffn_join_gradients_kernel(TileArgs sum, TileArgs pair, int sum_blocks) {
  const int block = blockIdx.x;
  if (block < sum_blocks) join<kSum, ISOLOCO_ACT_SILU, F32>(sum, block);
  else join<kPair, ISOLOCO_ACT_SILU, F32>(pair, block - sum_blocks);
}

template <int MODE, class C>
TileArgs tile_args(const FfnArgs& g, int splits) {
  constexpr int kCols = MODE == kForward || MODE == kInner ? C::TN / 2 : C::TN;
  TileArgs t;
  t.g = g;
  t.planes = MODE == kPair ? 2 : 1;
  t.splits = splits;
  t.tiles_m = (int)((g.m + C::TM - 1) / C::TM);
  t.tiles_n = (int)((g.n + kCols - 1) / kCols);
  t.tiles = t.tiles_m * t.tiles_n * t.planes * t.splits;
  return t;
}

template <int MODE>
unsigned join_blocks(const TileArgs& t) {
  const int64_t quads = t.planes * (MODE == kInner ? ffn_pad(t.g.m) : t.g.m) * partial_cols(MODE, t.g) / 4;
  return t.splits > 1 ? (unsigned)((quads + 255) / 256) : 0;
}

template <int MODE, int ACT, bool F32, class C>
void launch_shape(const FfnArgs& g, int splits, hipStream_t st) {
  const TileArgs t = tile_args<MODE, C>(g, splits);
  hipLaunchKernelGGL((ffn_tile_kernel<MODE, ACT, F32, C>), dim3(t.tiles), dim3(C::threads), 0, st, t);
  if (splits > 1)
    hipLaunchKernelGGL((ffn_join_kernel<MODE, ACT, F32>), dim3(join_blocks<MODE>(t)), dim3(256), 0, st, t);
}

template <int MODE, int ACT, bool F32>
hipError_t launch_mode(const FfnArgs& g, const Plan& p, hipStream_t st) {
  if (g.m == 0 || g.n == 0) return hipSuccess;
  if (p.shape == kLarge) launch_shape<MODE, ACT, F32, Large>(g, p.splits, st);
  else if (p.shape == kMiddle) launch_shape<MODE, ACT, F32, Middle>(g, p.splits, st);
  else launch_shape<MODE, ACT, F32, Small>(g, p.splits, st);
  return hipGetLastError();
}

template <bool F32>
hipError_t launch_projections(FfnMode mode, int act, const FfnArgs& g, hipStream_t st) {
  const Plan p = plan_of(mode, F32, g.m, g.n, g.k);
  if (mode == kForward)
    return act == ISOLOCO_ACT_SILU ? launch_mode<kForward, ISOLOCO_ACT_SILU, F32>(g, p, st)
                                   : launch_mode<kForward, ISOLOCO_ACT_GELU, F32>(g, p, st);
  return act == ISOLOCO_ACT_SILU ? launch_mode<kInner, ISOLOCO_ACT_SILU, F32>(g, p, st)
                                 : launch_mode<kInner, ISOLOCO_ACT_GELU, F32>(g, p, st);
}

template <bool F32, class CS, class CP>
hipError_t launch_together(const FfnArgs& sum, const FfnArgs& pair, const GradientsPlan& p, hipStream_t st) {
  FfnArgs after = pair;
  after.partial += partial_bytes(p.sum, kSum, sum.m, sum.n) / sizeof(float);
  const TileArgs s = tile_args<kSum, CS>(sum, p.sum.splits), q = tile_args<kPair, CP>(after, p.pair.splits);
  hipLaunchKernelGGL((ffn_gradients_kernel<F32, CS, CP>), dim3(s.tiles + q.tiles), dim3(CS::threads), 0, st, s, q);
  const unsigned js = join_blocks<kSum>(s), jq = join_blocks<kPair>(q);
  if (js + jq) hipLaunchKernelGGL(ffn_join_gradients_kernel<F32>, dim3(js + jq), dim3(256), 0, st, s, q, (int)js);
  return hipGetLastError();
}

// (these two apply no activation)  One of them alone goes by the same plan: the same bits.
template <bool F32>
hipError_t launch_gradients(const FfnArgs* sum, const FfnArgs* pair, hipStream_t st) {
  if (!sum && !pair) return hipSuccess;
  const GradientsPlan p =
      sum ? plan_gradients(F32, sum->m, sum->n, sum->k) : plan_gradients(F32, pair->k, pair->n, pair->m);
  if (sum && pair && p.together) {
    if (p.sum.shape == kSmall) return launch_together<F32, Small, Small>(*sum, *pair, p, st);
    if (p.pair.shape == kLarge) return launch_together<F32, Large, Large>(*sum, *pair, p, st);
    return launch_together<F32, Large, Middle>(*sum, *pair, p, st);
  }
  hipError_t e = hipSuccess;
  if (sum) e = launch_mode<kSum, ISOLOCO_ACT_SILU, F32>(*sum, p.sum, st);
  if (e == hipSuccess && pair) e = launch_mode<kPair, ISOLOCO_ACT_SILU, F32>(*pair, p.pair, st);
  return e;
}

}  // namespace

size_t ffn_projections_partial_bytes(FfnMode mode, bool f32, int64_t m, int64_t n, int64_t k) {
  return partial_bytes(plan_of(mode, f32, m, n, k), mode, m, n);
}

size_t ffn_gradients_partial_bytes(bool f32, int64_t m, int64_t n, int64_t k) {
  const GradientsPlan p = plan_gradients(f32, m, n, k);
  const size_t sum = partial_bytes(p.sum, kSum, m, n), pair = partial_bytes(p.pair, kPair, k, n);
  return p.together ? sum + pair : std::max(sum, pair);
}

hipError_t launch_ffn_projections(FfnMode mode, int act, bool f32, const FfnArgs& g, hipStream_t st) {
  return f32 ? launch_projections<true>(mode, act, g, st) : launch_projections<false>(mode, act, g, st);
}

hipError_t launch_ffn_gradients(bool f32, const FfnArgs* sum, const FfnArgs* pair, hipStream_t st) {
  return f32 ? launch_gradients<true>(sum, pair, st) : launch_gradients<false>(sum, pair, st);
}

}  // namespace isoloco
