// Rows of float32 or bfloat16 values, 16 bytes at a time.
#pragma once
#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include "isoloco_device.h"

namespace isoloco {

// 16 bytes at the alignment of an element: the hardware takes such accesses whole.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr float kLog2e = 1.44269504088896340736f;

// scale log2 e, finite: 0 times it stays 0
__host__ __device__ inline float rate_of(float scale) { return fminf(scale * kLog2e, FLT_MAX); }

template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
};
template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float* x) {
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

template <typename T>
__device__ __forceinline__ u32x4 pack(const float* x) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
      v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){x[2 * i], x[2 * i + 1]}, bf16x2_t));
    } else {
      v[i] = __float_as_uint(x[i]);
    }
  }
  return v;
}

// 4 values as bfloat16
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ u32x2_any pack4(const float* x) {
  typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
  typedef float floatx4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2_any, __builtin_convertvector((floatx4_t){x[0], x[1], x[2], x[3]}, bf16x4_t));
}

// The order of the values: of equal ones (-0 and 0 among them) the lower index is
// the larger key; NaN is above all.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xffffffffu : ((u >> 31) ? ~u : (u | 0x80000000u));
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) {
  return ((uint64_t)order_of(x) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u);
}
__device__ __forceinline__ int64_t index_of(uint64_t key) { return (int64_t)(uint32_t)~(uint32_t)key; }
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// The first `left` values of a row's piece of 16 bytes as they are stored, zeros after them.
// PAST: of data that is read once and larger than the caches.
template <typename T, bool PAST = false>
__device__ __forceinline__ u32x4 load_raw(const T* p, int64_t left) {
  if (left >= Vec<T>::N) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
    return *reinterpret_cast<const u32x4_any*>(p);
  }
  float x[Vec<T>::N];
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) x[e] = e < left ? (float)p[e] : 0.f;
  return pack<T>(x);
}
template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int64_t left, float* x) {
  unpack<T>(load_raw<T>(p, left), x);
}
template <typename T, bool PAST = false>
__device__ __forceinline__ void store_piece(T* p, int64_t left, const float* x) {
  if (left >= Vec<T>::N) {
    if constexpr (PAST) __builtin_nontemporal_store(pack<T>(x), reinterpret_cast<u32x4_any*>(p));
    else *reinterpret_cast<u32x4_any*>(p) = pack<T>(x);
  } else {
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
      if (e < left) p[e] = (T)x[e];
  }
}

// Indices of 32 or 64 bits.
struct Index {
  const void* p;
  bool wide;
  __device__ __forceinline__ int64_t get(int64_t i) const {
    return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
  }
};

}  // namespace isoloco
