// Failure reporting and argument checks of the C ABI's entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "isoloco.h"

namespace isoloco {

// Keep the message for isoloco_last_error() of this thread and return s.
isoloco_status fail(isoloco_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
isoloco_status hip_fail(hipError_t e, const char* what);

inline bool is_dtype(int32_t d) { return d == ISOLOCO_F32 || d == ISOLOCO_BF16; }
inline size_t dtype_bytes(int32_t d) { return d == ISOLOCO_F32 ? 4 : 2; }
inline bool is_index_type(int32_t t) { return t == ISOLOCO_I32 || t == ISOLOCO_I64; }
inline size_t index_bytes(int32_t t) { return t == ISOLOCO_I32 ? 4 : 8; }

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The bytes of a rows x cols matrix of `elem` bytes whose rows start ld elements
// apart (no rows or columns: none).
inline size_t matrix_bytes(int64_t rows, int64_t cols, int64_t ld, size_t elem) {
  return rows <= 0 || cols <= 0 ? 0 : ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem;
}

inline bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na && nb && x < y + nb && y < x + na;
}

// Sizes the operators accept: any product of two of them stays below 2^62.
constexpr int64_t kMaxExtent = (int64_t)1 << 31;

// A launch's threads are counted in 32 bits.
inline bool launchable(int64_t blocks, int threads) { return blocks <= (int64_t)UINT32_MAX / threads; }

// The card's last cache.  A result that is larger is stored past the caches: its reader
// would not find it there, and what is there stays.
constexpr int64_t kCacheBytes = (int64_t)256 << 20;

#define ISOLOCO_TRY(expr)                          \
  do {                                             \
    const isoloco_status try_status_ = (expr);     \
    if (try_status_ != ISOLOCO_OK) return try_status_; \
  } while (0)

// A matrix operand: not NULL unless empty, its rows at least cols apart, its
// start aligned to its elements.
inline isoloco_status check_matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld,
                                   size_t elem) {
  if (rows == 0) return ISOLOCO_OK;
  if (!p) return fail(ISOLOCO_ERR_INVALID_ARG, "%s is NULL", name);
  if (ld < cols || ld > kMaxExtent)
    return fail(ISOLOCO_ERR_INVALID_ARG, "%s: rows %lld elements apart, of %lld elements", name, (long long)ld,
                (long long)cols);
  if (!aligned_to(p, elem)) return fail(ISOLOCO_ERR_ALIGN, "%s is not aligned to its %zu-byte elements", name, elem);
  return ISOLOCO_OK;
}

inline isoloco_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return ISOLOCO_OK;
  if (!ws || have < need) return fail(ISOLOCO_ERR_WORKSPACE, "workspace of %zu bytes, %zu are needed", ws ? have : 0, need);
  if (!aligned_to(ws, 256)) return fail(ISOLOCO_ERR_WORKSPACE, "the workspace is not 256-byte aligned");
  return ISOLOCO_OK;
}

struct Operand {
  const char* name;
  const void* p;
  size_t bytes, align;
};

// Operands of a call: inputs and outputs not NULL unless empty, aligned to their elements,
// outputs apart from inputs and from each other.
inline isoloco_status check_operands(const Operand* outs, int n_out, const Operand* ins, int n_in) {
  for (int i = 0; i < n_in; ++i) {
    if (ins[i].bytes && !ins[i].p) return fail(ISOLOCO_ERR_INVALID_ARG, "%s is NULL", ins[i].name);
    if (!aligned_to(ins[i].p, ins[i].align)) return fail(ISOLOCO_ERR_ALIGN, "%s is not aligned to its elements", ins[i].name);
  }
  for (int i = 0; i < n_out; ++i) {
    if (outs[i].bytes && !outs[i].p) return fail(ISOLOCO_ERR_INVALID_ARG, "%s is NULL", outs[i].name);
    if (!aligned_to(outs[i].p, outs[i].align)) return fail(ISOLOCO_ERR_ALIGN, "%s is not aligned to its elements", outs[i].name);
    for (int j = 0; j < n_in; ++j)
      if (ranges_overlap(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes))
        return fail(ISOLOCO_ERR_ALIAS, "%s overlaps %s", outs[i].name, ins[j].name);
    for (int j = 0; j < i; ++j)
      if (ranges_overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
        return fail(ISOLOCO_ERR_ALIAS, "%s overlaps %s", outs[i].name, outs[j].name);
  }
  return ISOLOCO_OK;
}

}  // namespace isoloco
