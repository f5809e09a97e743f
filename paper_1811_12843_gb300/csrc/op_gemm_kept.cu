// The products that keep their pre-activations as a checkpoint (op_gemm_kernel.cuh): kernels of their own, since beside
// the other results these cost registers.
#include "op_gemm_kernel.cuh"

namespace lipz {
namespace ops {

cudaError_t run_kept_product(const GemmPlan& plan, const Products& q, cudaStream_t st) {
  float* const parts[2] = {nullptr, nullptr};
  return q.g[0].type == LIPZ_E4M3 ? launch_shape<LIPZ_E4M3, true, 1>(q, plan, parts, nullptr, st)
                                  : launch_shape<LIPZ_BF16, true, 1>(q, plan, parts, nullptr, st);
}

}  // namespace ops
}  // namespace lipz
