// What the tile products share: tile shapes, operands as slabs in LDS, results on their
// way out.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "isoloco_device.h"
#include "isoloco_ffn_plan.h"
#include "isoloco_lds.h"

namespace isoloco {

// A tile shape: TM x TN outputs per workgroup, WM x WN waves of 32 x 32 blocks.
template <int TM_, int TN_, int WM_, int WN_>
struct Shape {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;
  static constexpr int waves = WM * WN, threads = 64 * waves;
  static constexpr int NA = TM / WM / 32, NB = TN / WN / 32;
};
typedef Shape<256, 256, 4, 2> Large;
typedef Shape<192, 256, 2, 4> Middle;
typedef Shape<128, 128, 2, 2> Small;

// ROWS rows of an operand whose k values lie along its rows: 128 bytes of each.
// The 16-byte pieces of an LDS row are XORed with bits 1-3 of the row, so that a
// fragment read touches every bank once.
template <int ROWS, int THREADS>
struct RowsSlab {
  static constexpr int kBytes = ROWS * 128, kLoads = ROWS * 8 / THREADS;
  uint32_t vo[kLoads];
  __device__ static __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }
  __device__ static __forceinline__ int piece(int at) { return (at & 7) ^ swizzle(at >> 3); }
  // rows past the operand's are its last one again: their outputs are not stored
  __device__ __forceinline__ void init(uint32_t row_bytes, int64_t rows_left) {
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int at = q * THREADS + threadIdx.x;
      vo[q] = (uint32_t)min((int64_t)(at >> 3), rows_left - 1) * row_bytes + 16u * piece(at);
    }
  }
  __device__ __forceinline__ void load(uint32_t lds, const void* tile, int64_t slab) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32x4 r = tile_rsrc((uint64_t)tile + 128u * slab);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load_to_lds(lds + 16u * (q * THREADS + wave * 64), r, vo[q], 0);
  }
  // the last slab of an operand whose k values end inside it: zeros past them
  __device__ __forceinline__ void load_end(char* lds, const void* tile, int64_t slab, int k_left) const {
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int at = q * THREADS + threadIdx.x;
      u32x4 v = {};
      if (piece(at) * 8 < k_left)
        v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(tile) + 128 * slab + vo[q]);
      *reinterpret_cast<u32x4*>(lds + 16 * at) = v;
    }
  }
  // the same from a place that has `bytes` bytes: vo past them give zeros, as the k values
  // from k_left on do
  __device__ __forceinline__ void load(uint32_t lds, uint64_t place, uint32_t bytes, int64_t k_left) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32x4 r = tile_rsrc(place, bytes);
    if (k_left >= kSlab) {
#pragma unroll
      for (int q = 0; q < kLoads; ++q) load_to_lds(lds + 16u * (q * THREADS + wave * 64), r, vo[q], 0);
    } else {
#pragma unroll
      for (int q = 0; q < kLoads; ++q)
        load_to_lds(lds + 16u * (q * THREADS + wave * 64), r,
                    8 * piece(q * THREADS + (int)threadIdx.x) < k_left ? vo[q] : kOutside, 0);
    }
  }
  // 8 k values from k = kk + 8 (lane / 32) of row `row0 + lane % 32`
  __device__ static __forceinline__ bf16x8 frag(const char* lds, int row0, int kk) {
    const int lane = threadIdx.x & 63, p = ((kk >> 3) + (lane >> 5)) ^ swizzle(lane & 31);
    return *reinterpret_cast<const bf16x8*>(lds + (row0 + (lane & 31)) * 128 + p * 16);
  }
};

// COLS columns of an operand whose k values lie across its rows (row k of memory
// holds k's value of every column).  The fragments need k along a lane's registers:
// they are read with the transposing LDS load (16 lanes read 4 consecutive k of 16
// columns and receive a column's 4 values each).  The pieces of an LDS row are moved
// by 64 bytes times k mod 4, so that such a read touches every bank once.  (192 columns are
// no power of two: pieces go round the end of their row, and reads of the last 96 columns
// find two of them in a bank.)
template <int COLS, int THREADS>
struct ColsSlab {
  static constexpr int kRow = COLS * 2, kPieces = kRow / 16;
  static constexpr int kBytes = kSlab * kRow, kLoads = kBytes / 16 / THREADS;
  static constexpr bool kPow2 = (kPieces & (kPieces - 1)) == 0;
  uint32_t vo[kLoads];
  uint32_t row_bytes;
  // where piece p of row k lies, and which piece lies at p
  __device__ static __forceinline__ int place(int p, int k) {
    if constexpr (kPow2) return p ^ ((k & 3) << 2);
    p += (k & 3) << 2;
    return p >= kPieces ? p - kPieces : p;
  }
  __device__ static __forceinline__ int piece(int p, int k) {
    if constexpr (kPow2) return p ^ ((k & 3) << 2);
    p -= (k & 3) << 2;
    return p < 0 ? p + kPieces : p;
  }
  // columns past the operand's: its last 8 again (their outputs are not stored)
  __device__ __forceinline__ void init(uint32_t bytes, int64_t cols_left) {
    row_bytes = bytes;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int at = q * THREADS + threadIdx.x, k = at / kPieces;
      const int p = piece(at % kPieces, k);
      vo[q] = (uint32_t)k * row_bytes + 16u * (uint32_t)min((int64_t)p, cols_left / 8 - 1);
    }
  }
  // rows from k_left on are the last one again: the other operand is zero there
  __device__ __forceinline__ void load(uint32_t lds, const void* tile, int64_t slab, int64_t k_left) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32x4 r = tile_rsrc((uint64_t)tile + (uint64_t)(kSlab * slab) * row_bytes);
    if (k_left >= kSlab) {
#pragma unroll
      for (int q = 0; q < kLoads; ++q) load_to_lds(lds + 16u * (q * THREADS + wave * 64), r, vo[q], 0);
    } else {
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        const int k = (q * THREADS + (int)threadIdx.x) / kPieces;
        load_to_lds(lds + 16u * (q * THREADS + wave * 64), r,
                    vo[q] - (uint32_t)max(k - (int)k_left + 1, 0) * row_bytes, 0);
      }
    }
  }
  // the same from a place that has `bytes` bytes: rows past them give zeros
  __device__ __forceinline__ void load_bounded(uint32_t lds, uint64_t place, uint32_t bytes) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32x4 r = tile_rsrc(place, bytes);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load_to_lds(lds + 16u * (q * THREADS + wave * 64), r, vo[q], 0);
  }
  // 8 k values from k = kk + 8 (lane / 32) of column `col0 + lane % 32`
  __device__ static __forceinline__ bf16x8 frag(const char* lds, int col0, int kk) {
    const int lane = threadIdx.x & 63, j = lane & 15, kq = j >> 2;
    const int p = place(col0 / 8 + ((lane >> 4) & 1) * 2 + ((j & 3) >> 1), kq);
    const char* at = lds + (kk + 8 * (lane >> 5) + kq) * kRow + p * 16 + (j & 1) * 8;
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * kRow));
    return __builtin_shufflevector(__builtin_bit_cast(bf16x4, v0), __builtin_bit_cast(bf16x4, v1), 0, 1, 2, 3, 4, 5, 6,
                                   7);
  }
};

__device__ __forceinline__ bf16x4 rounded(floatx4 v) { return __builtin_convertvector(v, bf16x4); }

// A wave's LDS accesses before are done before those after.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 16 bytes at the alignment of an element: the hardware takes such accesses whole.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef floatx4 floatx4_any __attribute__((aligned(4)));

// A wave's 32 rows x COLS columns between LDS (rows of COLS * 2 + 16 bytes) and
// memory; rows and columns past the matrix are left out, those before `rows_pad`
// and `cols_pad` stored as zeros.
template <int COLS>
struct Patch {
  static constexpr int kPitch = COLS * 2 + 16, kBytes = 32 * kPitch, kLanes = COLS / 8, kRows = 64 / kLanes;
  __device__ static __forceinline__ char* quad(char* ws, int col) { return ws + (threadIdx.x & 31) * kPitch + col * 2; }
  __device__ static __forceinline__ void store(const char* ws, uint16_t* out, int64_t ld, int64_t row0, int64_t col0,
                                               int64_t rows, int64_t cols, int64_t rows_pad, int64_t cols_pad) {
    const int lane = threadIdx.x & 63, c8 = lane % kLanes;
    const int64_t col = col0 + 8 * c8;
#pragma unroll
    for (int q = 0; q < 32 / kRows; ++q) {
      const int r = q * kRows + lane / kLanes;
      const int64_t row = row0 + r;
      if (row >= rows_pad || col >= cols_pad) continue;
      uint16_t* o = out + row * ld + col;
      if (row < rows && col + 8 <= cols) {
        *reinterpret_cast<u32x4_any*>(o) = *reinterpret_cast<const u32x4*>(ws + r * kPitch + c8 * 16);
      } else {
        const uint16_t* v = reinterpret_cast<const uint16_t*>(ws + r * kPitch + c8 * 16);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < cols_pad) o[e] = row < rows && col + e < cols ? v[e] : (uint16_t)0;
      }
    }
  }
  u32x4 held[32 / kRows];
  __device__ __forceinline__ void fetch(const uint16_t* in, int64_t ld, int64_t row0, int64_t col0, int64_t rows,
                                        int64_t cols) {
    const int lane = threadIdx.x & 63, c8 = lane % kLanes;
    const int64_t col = col0 + 8 * c8;
#pragma unroll
    for (int q = 0; q < 32 / kRows; ++q) {
      const int64_t row = row0 + q * kRows + lane / kLanes;
      u32x4 v = {};
      const uint16_t* i = in + row * ld + col;
      if (row < rows) {
        if (col + 8 <= cols) {
          v = *reinterpret_cast<const u32x4_any*>(i);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < cols) v[e / 2] |= (uint32_t)i[e] << (16 * (e & 1));
        }
      }
      held[q] = v;
    }
  }
  __device__ __forceinline__ void put(char* ws) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < 32 / kRows; ++q)
      *reinterpret_cast<u32x4*>(ws + (q * kRows + lane / kLanes) * kPitch + (lane % kLanes) * 16) = held[q];
  }
};

// 4 consecutive float32 values, of which the first `left` exist
__device__ __forceinline__ floatx4 load4(const float* p, int64_t left) {
  if (left >= 4) return *reinterpret_cast<const floatx4_any*>(p);
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < left ? p[e] : 0.f;
  return v;
}
__device__ __forceinline__ void store4(float* p, floatx4 v, int64_t left) {
  if (left >= 4) {
    *reinterpret_cast<floatx4_any*>(p) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = v[e];
}

// The next bfloat16 part of 4 values, which keep the remainder (exact)
__device__ __forceinline__ bf16x4 next_part(floatx4& x) {
  const bf16x4 p = rounded(x);
  x -= __builtin_convertvector(p, floatx4);
  return p;
}

}  // namespace isoloco
