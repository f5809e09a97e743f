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

// Sums that a launch forms beside its products: out[g][c] = sum over p < parts of part[g][p][c], SUM_WAYS
// parts at a time.
constexpr int SUM_WAYS = 16;
struct PartSums {
  const float* part;
  int64_t cols;
  int groups, parts;
  lipz_vec out;
};

// One product, or two independent ones (the backward's: products with a plain epilogue and the same type
// of results), which then share a launch.
struct Products {
  Gemm g[2];
  int n;
};

// Copies of operands whose rows TMA does not take, to rows of whole 16-byte units.
struct RowCopy {
  const uint8_t* src;
  void* dst;
  int64_t group, ld, rows, total;  // strides in bytes; rows of a group, of all
  int64_t bytes, units;            // of a row: to copy; 16-byte units there
};

// How products will run: their scratch memory, and the copies that have to be made before them.
struct GemmPlan {
  struct One {
    int splits;
    bool copy_a, copy_b;
    int64_t tiles_m, tiles_n, chunks, chunks_per_split, lda, ldb, ldp;
    uint64_t a_bytes, b_bytes, part_bytes;
  } p[2];
  int cg, bn;
  bool direct;  // operands from rows that TMA does not take, without copies
  bool sums;    // results that are sums, in fp32 registers, of sums over a few chunks of k
  uint64_t bytes;
};
GemmPlan plan_products(const Products& q);
// The scratch memory of a plan (already part of plan_products' own).
void plan_space(const Products& q, GemmPlan* plan);
// The copies that the products of a plan need, into its workspace (copies[4]), and the operands that the
// products then have.
int plan_copies(const GemmPlan& plan, Products* q, void* workspace, RowCopy* copies);
constexpr int COPY_ROWS = 8;  // rows of a block
struct CopyJobs {
  RowCopy c[4];
  int n;
  int64_t blocks;
};
CopyJobs copy_jobs(const RowCopy* c, int n);
cudaError_t run_copies(const CopyJobs& jobs, cudaStream_t st);
// The products themselves; sums: null, or formed beside them.
cudaError_t run_products(const GemmPlan& plan, const Products& q, void* workspace, const PartSums* sums,
                         cudaStream_t st);

// The word that a kernel of this thread's calls sets when one of its waits expires (null: none can be had).
int* timeout_word();

}  // namespace ops
}  // namespace lipz
