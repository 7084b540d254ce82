// Loads from memory straight into LDS, and the waits that go with them.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "isoloco_device.h"

namespace isoloco {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16 bytes per lane from memory to LDS: lane l's bytes land at lds_off + 16 l
// (lds_off is wave-uniform).  No register receives the data; the loads count
// in vmcnt like any other, and wait_slabs() below waits for them.  m0 holds
// the LDS address.  It is listed as clobbered, so that the compiler sets it again
// for any use of its own (it has none here today); m0 is a reserved register,
// of which the compiler warns.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(uint32_t lds_off, u32x4 rsrc, uint32_t voff, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds_off), "v"(voff), "s"(rsrc), "s"(soff)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Wait until at most N of this wave's loads are outstanding and its LDS reads
// have returned, then for every wave of the workgroup.
template <int N>
__device__ __forceinline__ void wait_slabs() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A buffer of `bytes` bytes from base: loads at offsets past them give zeros.
__device__ __forceinline__ u32x4 tile_rsrc(uint64_t base, uint32_t bytes = 0xffffffffu) {
  u32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((uint32_t)base);
  r[1] = __builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xffffu);
  r[2] = __builtin_amdgcn_readfirstlane(bytes);
  r[3] = kBufferFlags;
  return r;
}

// An offset past any buffer of at most kMostBytes, that leaves room for 16 bytes and a slab's step
constexpr uint32_t kOutside = 0xfffff000u, kMostBytes = 0xffffe000u;

}  // namespace isoloco
