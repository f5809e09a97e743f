// The products that keep their pre-activations as a checkpoint (op_gemm_kernel.cuh): kernels of their own, since
// beside the other results these cost registers. They have 96 of them and spill themselves: per thread 208 bytes of stores
// and 584 of loads in 256 x 256 tiles (8 bits 224 and 648), in those of 128 columns 40 to 48 and 64 to 76 (where results
// leave by TMA none), beside fp32 results 140 to 148 and 100 to 120. Measured: 8192 x 4096 -> 8192 with SiLU 323 to 365 us (0.91 to 0.80 of cuBLAS's rate; the
// power limit, and six sums to a tile), 144 x 100 x 256 -> 512 with gelu 22 by itself (68 MB, 10 us; four chunks of k to
// a tile, whose results take longer than its operands).
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
