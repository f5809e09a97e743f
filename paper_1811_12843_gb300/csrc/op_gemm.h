// Tensor-core product of the residual-block operators: C[m][n] = sum_k A(m, k) B(n, k) per group, with
// the forward's epilogue.
#pragma once

#include "ops.h"

namespace lipz {
namespace ops {

// y = act(u) + residual, u = C x_scale[m] w_scale[n] + bias[n], pre = u.
struct Epilogue {
  lipz_mat y, residual, pre;
  lipz_vec x_scale, w_scale, bias;
  int act;
  float slope;
};

// An operand's matrix as it lies in memory: rows of adjacent elements, `ld` elements apart. k_major: a
// row per m (or n), its elements along k; else a row per k, its elements along m (or n).
struct Operand {
  const void* data;
  int64_t group, ld;
  bool k_major;
};

struct Gemm {
  Operand a, b;
  int type;  // of both operands
  int64_t groups, m, n, k;
  Epilogue e;
};

// Scratch bytes of a product: copies of operands whose rows TMA does not take, partial sums.
uint64_t gemm_workspace(const Gemm& g);
cudaError_t gemm(const Gemm& g, void* workspace, cudaStream_t st);

// The device word that a kernel sets when one of its waits expires (null: none can be had).
int* timeout_word();

}  // namespace ops
}  // namespace lipz
