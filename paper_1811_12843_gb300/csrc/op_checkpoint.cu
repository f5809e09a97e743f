// Rows to checkpoints (8 bits, a power of two per 16 columns) and back. Bound: HBM.
#include "ops.cuh"

namespace lipz {
namespace ops {

namespace {

constexpr int B = LIPZ_BLOCK;

struct BlocksArgs {
  lipz_mat m;  // x, or y
  lipz_blocks c;
  int64_t rows, dim, blocks, total;  // of a group; of a row; of all rows
  int act;
  float slope;
};

// A block per thread. VEC: whole 16-byte units on both sides, else element by element.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_checkpoint(const BlocksArgs p) {
  constexpr int E = VEC ? 16 / sizeof(T) : 1;
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / p.blocks, b = i - row * p.blocks, g = row / p.rows, r = row - g * p.rows;
    const T* x = (const T*)p.m.data + g * p.m.group + r * p.m.row + b * B;
    const int cols = (int)min(p.dim - b * B, (int64_t)B);
    float v[B];
#pragma unroll
    for (int j = 0; j < B; j += E) {
      if (j < cols) {
        load_vec<T, E>(x + j, v + j);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[j + e] = 0.f;
      }
    }
    uint32_t top = 0, w[4];
#pragma unroll
    for (int j = 0; j < B; ++j) top = max(top, magnitude(v[j]));
    const BlockScale s = block_scale(top);
    block_multiples<B>(v, s.inv, w);
    int8_t* q = p.c.data + g * p.c.group + r * p.c.row + b * B;
    if (VEC && cols == B) {
      *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < B; ++j)
        if (j < cols) q[j] = (int8_t)(w[j / 4] >> j % 4 * 8);
    }
    p.c.scale[g * p.c.scale_group + r * p.c.scale_row + b] = (uint8_t)s.byte;
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_restore(const BlocksArgs p) {
  constexpr int E = VEC ? 16 / sizeof(T) : 1;
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / p.blocks, b = i - row * p.blocks, g = row / p.rows, r = row - g * p.rows;
    const int8_t* q = p.c.data + g * p.c.group + r * p.c.row + b * B;
    const int cols = (int)min(p.dim - b * B, (int64_t)B);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (VEC && cols == B) w = __ldg(reinterpret_cast<const uint4*>(q));
    else w = bytes16((const uint8_t*)q, cols);
    const float unit = block_unit(__ldg(p.c.scale + g * p.c.scale_group + r * p.c.scale_row + b));
    float v[B];
    block_values(w.x, unit, v), block_values(w.y, unit, v + 4);
    block_values(w.z, unit, v + 8), block_values(w.w, unit, v + 12);
    with_act(p.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < B; ++j) v[j] = act_value<decltype(act)::value>(v[j], p.slope);
    });
    T* y = (T*)p.m.data + g * p.m.group + r * p.m.row + b * B;
#pragma unroll
    for (int j = 0; j < B; j += E)
      if (j < cols) store_vec<T, E>(y + j, v + j);
  }
}

BlocksArgs blocks_args(const lipz_mat& m, const lipz_blocks& c, int64_t groups, int64_t rows, int64_t dim) {
  const int64_t blocks = ceil_div(dim, B);
  return {m, c, rows, dim, blocks, groups * rows * blocks, LIPZ_ACT_NONE, 0.f};
}
// Whether rows are whole 16-byte units of both.
bool whole(const BlocksArgs& p, int64_t groups) {
  return p.dim % (16 / type_bytes(p.m.type)) == 0 && rows_aligned(p.m, groups, p.rows, 16) &&
         rows_aligned(bytes_of(p.c), groups, p.rows, 16);
}
dim3 grid_of(const BlocksArgs& p) {
  const int64_t want = ceil_div(p.total, 256), most = 8 * (int64_t)sm_count();
  return dim3((unsigned)(want < most ? want : most));
}

}  // namespace

cudaError_t checkpoint_rows(const lipz_checkpoint_rows_args& a, cudaStream_t st) {
  const BlocksArgs p = blocks_args(a.x, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  const bool vec = whole(p, a.groups);
  if (a.x.type == LIPZ_FP32)
    return vec ? launch_pdl(k_checkpoint<float, true>, grid_of(p), dim3(256), 0, st, p)
               : launch_pdl(k_checkpoint<float, false>, grid_of(p), dim3(256), 0, st, p);
  return vec ? launch_pdl(k_checkpoint<bf16, true>, grid_of(p), dim3(256), 0, st, p)
             : launch_pdl(k_checkpoint<bf16, false>, grid_of(p), dim3(256), 0, st, p);
}

cudaError_t restore_rows(const lipz_restore_rows_args& a, cudaStream_t st) {
  BlocksArgs p = blocks_args(a.y, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  p.act = a.act, p.slope = a.slope;
  const bool vec = whole(p, a.groups);
  if (a.y.type == LIPZ_FP32)
    return vec ? launch_pdl(k_restore<float, true>, grid_of(p), dim3(256), 0, st, p)
               : launch_pdl(k_restore<float, false>, grid_of(p), dim3(256), 0, st, p);
  return vec ? launch_pdl(k_restore<bf16, true>, grid_of(p), dim3(256), 0, st, p)
             : launch_pdl(k_restore<bf16, false>, grid_of(p), dim3(256), 0, st, p);
}

}  // namespace ops
}  // namespace lipz
