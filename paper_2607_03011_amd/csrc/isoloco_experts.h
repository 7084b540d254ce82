// The products grouped by expert, shared by their kernel files.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "isoloco.h"
#include "isoloco_experts_plan.h"
#include "isoloco_vec.h"

namespace isoloco {

// Where the experts' rows lie.
struct Groups {
  Index offsets;  // experts + 1
  int64_t rows;
  int experts;
  // Group e's rows, inside 0 .. rows whatever the offsets; group `experts` is the rows behind
  // the last expert's.
  __device__ __forceinline__ void rows_of(int e, int64_t& begin, int64_t& end) const {
    begin = e == 0 ? 0 : min(max(offsets.get(e), (int64_t)0), rows);
    end = e >= experts ? rows : max(begin, min(offsets.get(e + 1), rows));
  }
};

// The tile products.  Operands are bfloat16 (float32: kFfnParts parts each, part_a and part_b
// elements apart), 16-byte aligned, their rows' distances multiples of 8 and at most 2^22,
// their columns multiples of 8.
//   kOut  a: rows (or, with token, tokens) of k, b: n rows of k per expert;  out: rows x n
//   kDx   a: rows of k, b: k rows of n per expert;                           out: rows x n
//         (wide_out: of float32, whatever the operands are; past: those past the caches)
//   kDw   a: rows of m, b: rows (or, with token, tokens) of n;               out: m x n per expert
struct ExpertArgs {
  Groups groups;
  const uint16_t *a, *b;
  int64_t ld_a, ld_b, part_a, part_b, stride_b;
  Index token;        // p NULL: rows as they lie
  int64_t tokens;     // of the operand that token reads, whose tokens * ld is at most kMostBytes
  int64_t m, n, k;    // m: of kDw
  int64_t cols_a, cols_b;  // columns of the operands whose rows are k values: multiples of 8, at least m and n
  void* out;
  int64_t ld_out, stride_out;
  bool wide_out, past;
  float* partial;
};

// kOut of rows of k
size_t expert_out_partial_bytes(bool f32, int64_t rows, int64_t experts, int64_t n, int64_t k);
hipError_t launch_expert_out(bool f32, const ExpertArgs& g, hipStream_t st);

// kDx and kDw, either of which may be NULL; their `partial` is the same.
size_t expert_gradients_partial_bytes(bool f32, int64_t rows, int64_t experts, int64_t dim, int64_t cols);
hipError_t launch_expert_gradients(bool f32, const ExpertArgs* dx, const ExpertArgs* dw, hipStream_t st);

// out[t] = sum_j y[row[t, j]] of float32 rows of dim, rounded once to out's type (past: the rows lie
// past the caches)
hipError_t launch_rows_sum(const float* y, int64_t rows, int64_t dim, Index row, int64_t tokens, int top_k, bool f32,
                           bool past, void* out, int64_t ld_out, hipStream_t st);

}  // namespace isoloco
