// Internal interface of the residual-block operators (include/lipz.h): operators.cu checks a call's
// arguments and launches the kernels of op_norm.cu, op_linear.cu and op_gemm.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "lipz.h"

namespace lipz {
namespace ops {

inline int type_bytes(int type) { return type == LIPZ_FP32 ? 4 : type == LIPZ_BF16 ? 2 : 1; }

// Whether every row of every matrix starts on a boundary of `bytes` (one row, one group: their strides
// are not used).
inline bool rows_aligned(const lipz_mat& m, int64_t groups, int64_t rows, int bytes) {
  uint64_t bits = (uint64_t)(uintptr_t)m.data;
  if (rows > 1) bits |= (uint64_t)m.row * type_bytes(m.type);
  if (groups > 1) bits |= (uint64_t)m.group * type_bytes(m.type);
  return bits % bytes == 0;
}
inline bool rows_aligned(const lipz_vec& v, int64_t groups, int bytes) {
  uint64_t bits = (uint64_t)(uintptr_t)v.data;
  if (groups > 1) bits |= (uint64_t)v.group * 4;
  return bits % bytes == 0;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// SMs of the current device.
int sm_count();

cudaError_t rmsnorm(const lipz_rmsnorm_args& a, cudaStream_t st);
// Parts per group in which the backward kernel's weight-gradient sums come; more than one go through the
// workspace, [groups][parts][dim] fp32.
int rmsnorm_backward_parts(const lipz_rmsnorm_backward_args& a);
cudaError_t rmsnorm_backward(const lipz_rmsnorm_backward_args& a, cudaStream_t st);
cudaError_t quantize_rows(const lipz_quantize_rows_args& a, cudaStream_t st);

// out[g][c] = sum over p < parts of part[g][p][c], in a fixed order: `ways` (at most 32) sums of every
// ways-th part, then theirs.
cudaError_t sum_parts(const float* part, int64_t groups, int parts, int64_t cols, lipz_vec out, int ways,
                      cudaStream_t st);

// Whether a call has the scratch memory that it needs.
inline bool space_given(const void* p, uint64_t have, uint64_t need) {
  return !need || (p && have >= need && (uintptr_t)p % 256 == 0);
}
// *need: the scratch memory; nothing is launched where the call does not have it. (The plan that tells is the
// launch's own. A caller that first asks for the size, as the torch binding does, has the plan made twice.)
uint64_t linear_workspace(const lipz_linear_args& a);
cudaError_t linear(const lipz_linear_args& a, cudaStream_t st, uint64_t* need);
uint64_t linear_backward_workspace(const lipz_linear_backward_args& a);
cudaError_t linear_backward(const lipz_linear_backward_args& a, cudaStream_t st, uint64_t* need);

}  // namespace ops
}  // namespace lipz
