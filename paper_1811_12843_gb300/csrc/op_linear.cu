// Matrix product with bias, activation and residual, and its backward pass.
#include <type_traits>

#include "ops.cuh"

namespace lipz {
namespace ops {

namespace {

// C[m][n] = sum_k A(m, k) B(n, k), one problem per group, with the forward's epilogue. Strides in
// elements along m or n and along k.
struct Product {
  const void *a, *b;
  int64_t ag, am, ak, bg, bn, bk;
  int64_t m, n, k;
  int ab_type;
  lipz_mat y, residual, pre;
  lipz_vec x_scale, w_scale, bias;
  int act;
  float slope;
};

__device__ __forceinline__ float element(const void* p, int64_t i, int type) {
  if (type == LIPZ_BF16) return __bfloat162float(reinterpret_cast<const bf16*>(p)[i]);
  __nv_fp8_e4m3 v;
  v.__x = reinterpret_cast<const e4m3*>(p)[i];
  return (float)v;
}

__global__ void __launch_bounds__(256) k_product(const Product p) {
  constexpr int BT = 64, BK = 16;
  __shared__ float sa[BK][BT + 1], sb[BK][BT + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * BT, n0 = (int64_t)blockIdx.x * BT, g = blockIdx.z;
  pdl_wait();
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < p.k; k0 += BK) {
    for (int i = threadIdx.x; i < BT * BK; i += 256) {
      const int ra = p.ak == 1 ? i / BK : i % BT, ka = p.ak == 1 ? i % BK : i / BT;
      const int rb = p.bk == 1 ? i / BK : i % BT, kb = p.bk == 1 ? i % BK : i / BT;
      sa[ka][ra] = m0 + ra < p.m && k0 + ka < p.k
                       ? element(p.a, g * p.ag + (m0 + ra) * p.am + (k0 + ka) * p.ak, p.ab_type) : 0.f;
      sb[kb][rb] = n0 + rb < p.n && k0 + kb < p.k
                       ? element(p.b, g * p.bg + (n0 + rb) * p.bn + (k0 + kb) * p.bk, p.ab_type) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < BK; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = fmaf(sa[kk][ty + 16 * i], sb[kk][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
  with_act(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
        if (m >= p.m || n >= p.n) continue;
        float u = acc[i][j];
        if (p.x_scale.data)
          u *= p.x_scale.data[g * p.x_scale.group + m] * p.w_scale.data[g * p.w_scale.group + n];
        if (p.bias.data) u += p.bias.data[g * p.bias.group + n];
        if (p.pre.data)
          reinterpret_cast<bf16*>(p.pre.data)[g * p.pre.group + m * p.pre.row + n] =
              __float2bfloat16_rn(u);
        float y = act_value<decltype(act)::value>(u, p.slope);
        const int64_t ro = g * p.residual.group + m * p.residual.row + n;
        const int64_t yo = g * p.y.group + m * p.y.row + n;
        if (p.residual.data)
          y += p.y.type == LIPZ_FP32 ? reinterpret_cast<const float*>(p.residual.data)[ro]
                                     : __bfloat162float(reinterpret_cast<const bf16*>(p.residual.data)[ro]);
        if (p.y.type == LIPZ_FP32) reinterpret_cast<float*>(p.y.data)[yo] = y;
        else reinterpret_cast<bf16*>(p.y.data)[yo] = __float2bfloat16_rn(y);
      }
  });
}

cudaError_t product(const Product& p, int64_t groups, cudaStream_t st) {
  return launch_pdl(k_product,
                    dim3((unsigned)ceil_div(p.n, 64), (unsigned)ceil_div(p.m, 64), (unsigned)groups),
                    dim3(256), 0, st, p);
}

// du = dy act'(pre), in bf16 rows of ldu elements, and the sums of its columns over the block's rows:
// 32 vectors of columns by 8 rows at a time. Bound: HBM.
struct DuArgs {
  lipz_mat dy, pre;
  bf16* du;     // [groups][rows][ldu], or null: the sums only
  float* part;  // [groups][gridDim.y][n], or null: no sums
  int64_t rows, n, ldu, rows_per_block;
  int act;
  float slope;
};

template <int E>
__global__ void __launch_bounds__(256) k_du(const DuArgs p) {
  __shared__ float s[8][32 * E + 1];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int64_t c = ((int64_t)blockIdx.x * 32 + tx) * E, g = blockIdx.z;
  const int64_t r0 = blockIdx.y * p.rows_per_block;
  const int64_t r1 = min(p.rows, r0 + p.rows_per_block);
  pdl_wait();
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  with_act(p.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if (c < p.n) {
#pragma unroll 4
      for (int64_t r = r0 + ty; r < r1; r += 8) {
        float d[E];
        load_vec<bf16, E>((const bf16*)p.dy.data + g * p.dy.group + r * p.dy.row + c, d);
        if constexpr (ACT != LIPZ_ACT_NONE) {
          float u[E];
          load_vec<bf16, E>((const bf16*)p.pre.data + g * p.pre.group + r * p.pre.row + c, u);
#pragma unroll
          for (int e = 0; e < E; ++e) d[e] *= act_slope<ACT>(u[e], p.slope);
        }
        if (p.du) store_vec<bf16, E>(p.du + (g * p.rows + r) * p.ldu + c, d);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += d[e];
      }
    }
  });
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < E; ++e) s[ty][tx * E + e] = sum[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * E; i += 256) {
    const int64_t col = (int64_t)blockIdx.x * 32 * E + i;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) v += s[q][i];
    if (col < p.n) p.part[(g * gridDim.y + blockIdx.y) * p.n + col] = v;
  }
}

// The workspace of a backward call: du, then the parts of db.
struct BackPlan {
  bool vec, need_du;
  int64_t ldu, blocks, rows_per_block;
  uint64_t du_bytes, bytes;
};
BackPlan back_plan(const lipz_linear_backward_args& a) {
  BackPlan b;
  b.vec = a.n % 8 == 0 && rows_aligned(a.dy, a.groups, a.rows, 16) &&
          (!a.pre.data || rows_aligned(a.pre, a.groups, a.rows, 16));
  b.need_du = a.act != LIPZ_ACT_NONE && (a.dx.data || a.dw.data);
  b.ldu = ceil_div(a.n, 8) * 8;
  // enough blocks to fill the device, of 8 rows or more
  const int64_t cols = ceil_div(a.n, b.vec ? 256 : 32), fill = 8 * sm_count();
  const int64_t want = ceil_div(fill, cols * (a.groups > 0 ? a.groups : 1));
  b.rows_per_block = ceil_div(ceil_div(a.rows > 0 ? a.rows : 1, want), 8) * 8;
  b.blocks = ceil_div(a.rows, b.rows_per_block);
  b.du_bytes = b.need_du ? ceil_div(a.groups * a.rows * b.ldu * 2, 256) * 256 : 0;
  b.bytes = b.du_bytes + (a.db.data ? (uint64_t)(a.groups * b.blocks * a.n * 4) : 0);
  return b;
}

}  // namespace

uint64_t linear_workspace(const lipz_linear_args&) { return 0; }

cudaError_t linear(const lipz_linear_args& a, cudaStream_t st) {
  if (a.groups == 0 || a.rows == 0) return cudaSuccess;
  Product p{a.x.data, a.w.data, a.x.group, a.x.row, 1, a.w.group, a.w.row, 1, a.rows, a.n, a.k,
            a.x.type, a.y, a.residual, a.pre, a.x_scale, a.w_scale, a.bias, a.act, a.slope};
  if (a.x.type != LIPZ_E4M3) p.x_scale.data = nullptr;
  return product(p, a.groups, st);
}

uint64_t linear_backward_workspace(const lipz_linear_backward_args& a) { return back_plan(a).bytes; }

cudaError_t linear_backward(const lipz_linear_backward_args& a, cudaStream_t st) {
  if (a.groups == 0) return cudaSuccess;
  if (a.rows == 0) {  // sums over no rows
    cudaError_t e = cudaSuccess;
    const int64_t row_bytes = a.k * type_bytes(a.dw.type);
    for (int64_t g = 0; g < a.groups && e == cudaSuccess; ++g) {
      if (a.dw.data)
        e = cudaMemset2DAsync((char*)a.dw.data + g * a.dw.group * type_bytes(a.dw.type),
                              a.n > 1 ? a.dw.row * type_bytes(a.dw.type) : row_bytes, 0, row_bytes,
                              a.n, st);
      if (a.db.data && e == cudaSuccess)
        e = cudaMemsetAsync(a.db.data + g * a.db.group, 0, a.n * 4, st);
    }
    return e;
  }
  const BackPlan b = back_plan(a);
  bf16* du = b.need_du ? (bf16*)a.workspace : nullptr;
  float* part = a.db.data ? (float*)((char*)a.workspace + b.du_bytes) : nullptr;
  cudaError_t e = cudaSuccess;
  if (du || part) {
    const DuArgs p{a.dy, a.pre, du, part, a.rows, a.n, b.ldu, b.rows_per_block, a.act, a.slope};
    const dim3 grid((unsigned)ceil_div(a.n, b.vec ? 256 : 32), (unsigned)b.blocks, (unsigned)a.groups);
    e = b.vec ? launch_pdl(k_du<8>, grid, dim3(256), 0, st, p)
              : launch_pdl(k_du<1>, grid, dim3(256), 0, st, p);
    if (e == cudaSuccess && part) e = sum_parts(part, a.groups, (int)b.blocks, a.n, a.db, st);
  }
  const void* d = du ? du : a.dy.data;
  const int64_t dg = du ? a.rows * b.ldu : a.dy.group, dr = du ? b.ldu : a.dy.row;
  if (e == cudaSuccess && a.dx.data) {
    Product p{d, a.w.data, dg, dr, 1, a.w.group, 1, a.w.row, a.rows, a.k, a.n, LIPZ_BF16, a.dx};
    e = product(p, a.groups, st);
  }
  if (e == cudaSuccess && a.dw.data) {
    Product p{d, a.x.data, dg, 1, dr, a.x.group, 1, a.x.row, a.n, a.k, a.rows, LIPZ_BF16, a.dw};
    e = product(p, a.groups, st);
  }
  return e;
}

}  // namespace ops
}  // namespace lipz
