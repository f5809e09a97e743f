// Rows to checkpoints (8 bits, a power of two per 16 columns) and back.
//
//     e = max(-126, the smallest with max |v| < 127.5 2^e over 16 columns),  data = v 2^-e to the nearest whole number
//
// The power comes from the largest magnitude's bits, so that dividing by it is exact, and multiples are found by one
// addition whose last bit is 1. A multiple of 8 bits times a power of two is a bf16 number: nothing is rounded on the
// way back. Bound: HBM; with an activation its exponential beside it (16384 x 4096, gelu, back: 40 us, without 35).
#include "ops.cuh"

namespace lipz {
namespace ops {

namespace {

constexpr int B = LIPZ_BLOCK;

struct BlocksArgs {
  lipz_mat m;  // x, or y
  lipz_blocks c;
  int64_t rows, dim, blocks, total;  // of a group; pieces of work of a row; of all rows
  int act;
  float slope;
  bool few;  // total below 2^31: the two divisors
  Divisor by_row, by_group;
};
struct At {
  int64_t g, r, b;
};
__device__ __forceinline__ At block_at(const BlocksArgs& p, int64_t i) {
  if (p.total == p.blocks) return {0, 0, i};
  if (p.few) {
    const int row = p.by_row((int)i), g = p.by_group(row);
    return {g, row - g * p.rows, (int)i - (int64_t)row * p.blocks};
  }
  const int64_t row = i / p.blocks, g = row / p.rows;
  return {g, row - g * p.rows, i - row * p.blocks};
}

// A block per thread and turn, in few registers: what keeps enough loads in flight is threads. (16384 x 4096 in bf16,
// 205 MB, to a checkpoint 32.8 us and back 34.6, 0.92 and 0.87 of the copy rate; two blocks at a time 32.1 and 39.3,
// four 33.4 and 47.7.) WIDE: 32 bytes of x at a time; SHIFT: its rows begin anywhere, and a block's elements come from
// the 16-byte units that hold them, moved by whole words and half words.
template <typename T, bool WIDE, bool SHIFT>
__global__ void __launch_bounds__(256) k_checkpoint(const BlocksArgs p) {
  constexpr int W = B * sizeof(T) / 4, U = 16 / sizeof(T);  // words of a block, elements of a unit
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * 256) {
    const At at = block_at(p, i);
    const T* src = (const T*)p.m.data + at.g * p.m.group + at.r * p.m.row + at.b * B;
    const int64_t left = p.dim - at.b * B;
    const int cols = left < B ? (int)left : B;
    uint32_t x[W + (SHIFT ? 4 : 0)];
    if constexpr (SHIFT) {
      const int m = (int)((uint64_t)src & 15) / (int)sizeof(T);  // elements of the first unit before the block
      const uint4* units = reinterpret_cast<const uint4*>((uint64_t)src & ~15ull);
#pragma unroll
      for (int j = 0; j <= W / 4; ++j) {
        const uint4 r = j * U < m + cols ? __ldg(units + j) : make_uint4(0, 0, 0, 0);
        x[4 * j] = r.x, x[4 * j + 1] = r.y, x[4 * j + 2] = r.z, x[4 * j + 3] = r.w;
      }
      const int words = sizeof(T) == 4 ? m : m >> 1;
#pragma unroll
      for (int j = 0; j < W + 2; ++j) x[j] = words & 2 ? x[j + 2] : x[j];
#pragma unroll
      for (int j = 0; j < W + 1; ++j) x[j] = words & 1 ? x[j + 1] : x[j];
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < W; ++j) x[j] = __funnelshift_r(x[j], x[j + 1], (m & 1) * 16);
      }
      if (cols < B) {  // (what lies behind the row is nothing of it)
#pragma unroll
        for (int e = 0; e < B; ++e)
          if (e >= cols) {
            if constexpr (sizeof(T) == 4) x[e] = 0;
            else x[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
          }
      }
    } else if (cols == B) {
#pragma unroll
      for (int j = 0; j < W; j += 8) load32<WIDE>((const char*)src + 4 * j, x + j);
    } else {  // (a row's last block, in 16-byte units)
#pragma unroll
      for (int j = 0; j < W; j += 4) {
        const uint4 r = j / 4 * U < cols ? *reinterpret_cast<const uint4*>((const char*)src + 4 * j)
                                         : make_uint4(0, 0, 0, 0);
        x[j] = r.x, x[j + 1] = r.y, x[j + 2] = r.z, x[j + 3] = r.w;
      }
    }
    float v[B], most = 0.f;
#pragma unroll
    for (int e = 0; e < B; ++e) {
      if constexpr (sizeof(T) == 4) v[e] = __uint_as_float(x[e]);
      else v[e] = __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
      most = max_nan(most, fabsf(v[e]));
    }
    const BlockScale s = block_scale(__float_as_uint(most));
    uint32_t w[4];
    block_multiples<B>(v, s.inv, w);
    int8_t* q = p.c.data + at.g * p.c.group + at.r * p.c.row + at.b * B;
    if (cols == B && (!SHIFT || ((uint64_t)q & 15) == 0)) {
      *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < B; ++e)
        if (e < cols) q[e] = (int8_t)(w[e / 4] >> e % 4 * 8);
    }
    p.c.scale[at.g * p.c.scale_group + at.r * p.c.scale_row + at.b] = (uint8_t)s.byte;
  }
}

template <typename T>
__device__ __forceinline__ void act_words(int act, float slope, float* v, uint32_t* w) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int j = 0; j < B; j += 2) act_pair<decltype(a)::value, sizeof(T) == 4>(v[j], v[j + 1], slope);
  });
#pragma unroll
  for (int j = 0; j < B * (int)sizeof(T) / 4; ++j) {
    if constexpr (sizeof(T) == 4) {
      w[j] = __float_as_uint(v[j]);
    } else {
      const __nv_bfloat162 r = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&r);
    }
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_restore(const BlocksArgs p) {
  constexpr int W = B * sizeof(T) / 4, U = 16 / sizeof(T);
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * 256) {
    const At at = block_at(p, i);
    const int8_t* src = p.c.data + at.g * p.c.group + at.r * p.c.row + at.b * B;
    const int64_t left = p.dim - at.b * B;
    const uint4 q = left >= B ? __ldg(reinterpret_cast<const uint4*>(src)) : bytes16((const uint8_t*)src, left);
    const float unit = block_unit(__ldg(p.c.scale + at.g * p.c.scale_group + at.r * p.c.scale_row + at.b));
    float v[B];
    block_values(q.x, unit, v), block_values(q.y, unit, v + 4);
    block_values(q.z, unit, v + 8), block_values(q.w, unit, v + 12);
    uint32_t w[W];
    act_words<T>(p.act, p.slope, v, w);
    T* y = (T*)p.m.data + at.g * p.m.group + at.r * p.m.row + at.b * B;
    if (left >= B) {
#pragma unroll
      for (int j = 0; j < W; j += 8) store32<WIDE>((char*)y + 4 * j, w + j);
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 4)
        if (j / 4 * U < left)
          *reinterpret_cast<uint4*>((char*)y + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
    }
  }
}

// The same where rows are off that grid: 16 columns from a 16-byte boundary of y on (a row's first and last in part),
// which are of two blocks.
template <typename T>
__global__ void __launch_bounds__(256) k_restore_shift(const BlocksArgs p) {
  constexpr int W = B * sizeof(T) / 4;
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * 256) {
    const At at = block_at(p, i);
    T* row = (T*)p.m.data + at.g * p.m.group + at.r * p.m.row;
    const int m = (int)((uint64_t)row & 15) / (int)sizeof(T);
    const int64_t col = at.b * B - m;  // of the first of the 16; it lies m columns before a block's border
    if (col >= p.dim) continue;
    const uint8_t* src = (const uint8_t*)p.c.data + at.g * p.c.group + at.r * p.c.row;
    const uint8_t* scale = p.c.scale + at.g * p.c.scale_group + at.r * p.c.scale_row;
    const bool all = col >= 0 && col + B <= p.dim;
    uint32_t q[4] = {0, 0, 0, 0};
    if (all) {
      const uint4 r = bytes16(src + col, B);
      q[0] = r.x, q[1] = r.y, q[2] = r.z, q[3] = r.w;
    } else {
#pragma unroll
      for (int e = 0; e < B; ++e)
        if (col + e >= 0 && col + e < p.dim) q[e / 4] |= (uint32_t)__ldg(src + col + e) << e % 4 * 8;
    }
    const float before = block_unit(at.b && m ? __ldg(scale + at.b - 1) : 0u);
    const float behind = block_unit(at.b * B < p.dim ? __ldg(scale + at.b) : 0u);
    float v[B];
#pragma unroll
    for (int j = 0; j < 4; ++j) block_values(q[j], 1.f, v + 4 * j);
#pragma unroll
    for (int e = 0; e < B; ++e) v[e] *= e < m ? before : behind;
    uint32_t w[W];
    act_words<T>(p.act, p.slope, v, w);
    if (all) {
#pragma unroll
      for (int j = 0; j < W; j += 4)
        *reinterpret_cast<uint4*>((char*)(row + col) + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < B; ++e)
        if (col + e >= 0 && col + e < p.dim) {
          if constexpr (sizeof(T) == 4) row[col + e] = __uint_as_float(w[e]);
          else reinterpret_cast<unsigned short*>(row)[col + e] = (unsigned short)(w[e >> 1] >> (e & 1) * 16);
        }
    }
  }
}

// Rows as `blocks` pieces of work each.
void share_out(BlocksArgs* p, int64_t groups, int64_t blocks) {
  p->blocks = blocks, p->total = groups * p->rows * blocks;
  p->few = p->total < INT32_MAX;
  if (p->few && p->total) p->by_row = divisor(blocks), p->by_group = divisor(p->rows);
}

// Rows that follow one another without gaps, in whole blocks, are one long row.
BlocksArgs blocks_args(const lipz_mat& m, const lipz_blocks& c, int64_t groups, int64_t rows, int64_t dim) {
  if (dim % B == 0 && (rows == 1 || (m.row == dim && c.row == dim && c.scale_row == dim / B)) &&
      (groups == 1 || (m.group == rows * dim && c.group == rows * dim && c.scale_group == rows * dim / B)))
    dim *= groups * rows, groups = rows = groups && rows;
  BlocksArgs p{m, c, rows, dim};
  share_out(&p, groups, ceil_div(dim, B));
  return p;
}
// Whether rows start on boundaries of `bytes` in m, and the checkpoint's on 16.
bool starts_on(const BlocksArgs& p, int64_t groups, int64_t rows, int bytes) {
  return rows_aligned(p.m, groups, rows, bytes) && rows_aligned(bytes_of(p.c), groups, rows, 16);
}
// Several waves of blocks, so that SMs that are ahead take more of them, each of several turns. (16384 x 4096, gelu, back:
// of 16 blocks per SM, six of them at a time, 41.2 us, of 48 39.8, of one turn each 41.2; fp32 with SiLU 55.9, 53.8, 53.3;
// to a checkpoint 33.9, 33.6, 35.1.)
dim3 grid_of(const BlocksArgs& p) {
  const int64_t want = ceil_div(p.total, 256), most = 48 * (int64_t)sm_count();
  return dim3((unsigned)(want < most ? want : most));
}

template <typename T>
cudaError_t checkpoint_of(const BlocksArgs& p, const lipz_checkpoint_rows_args& a, cudaStream_t st) {
  if (a.dim % (16 / sizeof(T)) || !starts_on(p, a.groups, a.rows, 16))
    return launch_pdl(k_checkpoint<T, false, true>, grid_of(p), dim3(256), 0, st, p);
  return starts_on(p, a.groups, a.rows, 32)
             ? launch_pdl(k_checkpoint<T, true, false>, grid_of(p), dim3(256), 0, st, p)
             : launch_pdl(k_checkpoint<T, false, false>, grid_of(p), dim3(256), 0, st, p);
}
template <typename T>
cudaError_t restore_of(BlocksArgs& p, const lipz_restore_rows_args& a, cudaStream_t st) {
  if (a.dim % (16 / sizeof(T)) || !starts_on(p, a.groups, a.rows, 16)) {
    share_out(&p, p.dim == a.dim ? a.groups : 1, ceil_div(p.dim + 16 / sizeof(T) - 1, B));
    return launch_pdl(k_restore_shift<T>, grid_of(p), dim3(256), 0, st, p);
  }
  return starts_on(p, a.groups, a.rows, 32) ? launch_pdl(k_restore<T, true>, grid_of(p), dim3(256), 0, st, p)
                                            : launch_pdl(k_restore<T, false>, grid_of(p), dim3(256), 0, st, p);
}

}  // namespace

cudaError_t checkpoint_rows(const lipz_checkpoint_rows_args& a, cudaStream_t st) {
  const BlocksArgs p = blocks_args(a.x, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  return a.x.type == LIPZ_FP32 ? checkpoint_of<float>(p, a, st) : checkpoint_of<bf16>(p, a, st);
}

cudaError_t restore_rows(const lipz_restore_rows_args& a, cudaStream_t st) {
  BlocksArgs p = blocks_args(a.y, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  p.act = a.act, p.slope = a.slope;
  return a.y.type == LIPZ_FP32 ? restore_of<float>(p, a, st) : restore_of<bf16>(p, a, st);
}

}  // namespace ops
}  // namespace lipz
