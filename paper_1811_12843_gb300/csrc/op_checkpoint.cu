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
  bool few;  // total below 2^31: the two divisors
  Divisor by_row, by_group;
};
struct At {
  int64_t g, r, b;
};
__device__ __forceinline__ At block_at(const BlocksArgs& p, int64_t i) {
  if (p.few) {
    const int row = p.by_row((int)i), g = p.by_group(row);
    return {g, row - g * p.rows, (int)i - (int64_t)row * p.blocks};
  }
  const int64_t row = i / p.blocks, g = row / p.rows;
  return {g, row - g * p.rows, i - row * p.blocks};
}

// A block per thread, AHEAD of them at a time, over whole 16-byte units on both sides; WIDE: and 32 bytes of x (y).
template <typename T>
constexpr int BLOCKS_AHEAD = sizeof(T) == 4 ? 2 : 4;

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_checkpoint(const BlocksArgs p) {
  constexpr int W = B * sizeof(T) / 4, AHEAD = BLOCKS_AHEAD<T>;  // words of a block
  pdl_wait();
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < p.total; i0 += AHEAD * step) {
    uint32_t x[AHEAD][W];
    At at[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
#pragma unroll
      for (int j = 0; j < W; ++j) x[a][j] = 0;
      if (i0 + a * step >= p.total) continue;
      at[a] = block_at(p, i0 + a * step);
      const T* src = (const T*)p.m.data + at[a].g * p.m.group + at[a].r * p.m.row + at[a].b * B;
      if (p.dim - at[a].b * B >= B) {
#pragma unroll
        for (int j = 0; j < W; j += 8) load32<WIDE>((const char*)src + 4 * j, x[a] + j);
      } else {  // (a row's last block, in 16-byte units)
#pragma unroll
        for (int j = 0; j < W; j += 4)
          if (at[a].b * B + j * 4 / (int)sizeof(T) < p.dim) {
            const uint4 r = *reinterpret_cast<const uint4*>((const char*)src + 4 * j);
            x[a][j] = r.x, x[a][j + 1] = r.y, x[a][j + 2] = r.z, x[a][j + 3] = r.w;
          }
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (i0 + a * step >= p.total) continue;
      float v[B], most = 0.f;
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(x[a][j]);
        else v[j] = __uint_as_float(j & 1 ? x[a][j >> 1] & 0xFFFF0000u : x[a][j >> 1] << 16);
        most = max_nan(most, fabsf(v[j]));
      }
      const BlockScale s = block_scale(__float_as_uint(most));
      uint32_t w[4];
      block_multiples<B>(v, s.inv, w);
      int8_t* q = p.c.data + at[a].g * p.c.group + at[a].r * p.c.row + at[a].b * B;
      const int64_t cols = p.dim - at[a].b * B;
      if (cols >= B) {
        *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int j = 0; j < B; j += 4)
          if (j < cols) *reinterpret_cast<uint32_t*>(q + j) = w[j / 4];
      }
      p.c.scale[at[a].g * p.c.scale_group + at[a].r * p.c.scale_row + at[a].b] = (uint8_t)s.byte;
    }
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_restore(const BlocksArgs p) {
  constexpr int W = B * sizeof(T) / 4, AHEAD = BLOCKS_AHEAD<T>;
  pdl_wait();
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < p.total; i0 += AHEAD * step) {
    uint4 q[AHEAD];
    uint32_t byte[AHEAD];
    At at[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      q[a] = make_uint4(0, 0, 0, 0), byte[a] = 0;
      if (i0 + a * step >= p.total) continue;
      at[a] = block_at(p, i0 + a * step);
      const int8_t* src = p.c.data + at[a].g * p.c.group + at[a].r * p.c.row + at[a].b * B;
      if (p.dim - at[a].b * B >= B) q[a] = __ldg(reinterpret_cast<const uint4*>(src));
      else q[a] = bytes16((const uint8_t*)src, p.dim - at[a].b * B);
      byte[a] = __ldg(p.c.scale + at[a].g * p.c.scale_group + at[a].r * p.c.scale_row + at[a].b);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (i0 + a * step >= p.total) continue;
      const float unit = block_unit(byte[a]);
      float v[B];
      block_values(q[a].x, unit, v), block_values(q[a].y, unit, v + 4);
      block_values(q[a].z, unit, v + 8), block_values(q[a].w, unit, v + 12);
      with_act(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < B; j += 2) act_pair<decltype(act)::value, sizeof(T) == 4>(v[j], v[j + 1], p.slope);
      });
      uint32_t w[W];
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if constexpr (sizeof(T) == 4) {
          w[j] = __float_as_uint(v[j]);
        } else {
          const __nv_bfloat162 r = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
          w[j] = *reinterpret_cast<const uint32_t*>(&r);
        }
      }
      T* y = (T*)p.m.data + at[a].g * p.m.group + at[a].r * p.m.row + at[a].b * B;
      if (p.dim - at[a].b * B >= B) {
#pragma unroll
        for (int j = 0; j < W; j += 8) store32<WIDE>((char*)y + 4 * j, w + j);
      } else {
#pragma unroll
        for (int j = 0; j < W; j += 4)
          if (at[a].b * B + j * 4 / (int)sizeof(T) < p.dim)
            *reinterpret_cast<uint4*>((char*)y + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
      }
    }
  }
}

// Rows off that grid: four lanes to a block, four columns to a lane, from the words that hold them.
constexpr int QUADS_AHEAD = 4;

template <typename T>
__global__ void __launch_bounds__(256) k_checkpoint_quads(const BlocksArgs p) {
  const int lane = threadIdx.x & 31, c = (lane & 3) * 4;
  const uint32_t four = 0xFu << (lane & 28);
  pdl_wait();
  const int64_t step = (int64_t)gridDim.x * 64;
  for (int64_t i0 = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2); i0 < p.total; i0 += QUADS_AHEAD * step) {
    uint32_t x[QUADS_AHEAD][sizeof(T)];
    At at[QUADS_AHEAD];
    int left[QUADS_AHEAD];  // columns of this lane
#pragma unroll
    for (int a = 0; a < QUADS_AHEAD; ++a) {
#pragma unroll
      for (int j = 0; j < (int)sizeof(T); ++j) x[a][j] = 0;
      left[a] = 0;
      if (i0 + a * step >= p.total) continue;
      at[a] = block_at(p, i0 + a * step);
      left[a] = (int)max((int64_t)0, min((int64_t)4, p.dim - at[a].b * B - c));
      const T* src = (const T*)p.m.data + at[a].g * p.m.group + at[a].r * p.m.row + at[a].b * B + c;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left[a]) x[a][j] = __ldg(reinterpret_cast<const uint32_t*>(src) + j);
      } else if (left[a] == 4) {
        const uint32_t off = (uint32_t)(uint64_t)src & 2u;
        const uint32_t* w = reinterpret_cast<const uint32_t*>((const char*)src - off);
        const uint32_t w0 = __ldg(w), w1 = __ldg(w + 1), w2 = off ? __ldg(w + 2) : 0u;
        x[a][0] = __funnelshift_r(w0, w1, off * 8), x[a][1] = __funnelshift_r(w1, w2, off * 8);
      } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(src);
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left[a]) x[a][j >> 1] |= (uint32_t)__ldg(h + j) << (j & 1) * 16;
      }
    }
#pragma unroll
    for (int a = 0; a < QUADS_AHEAD; ++a) {
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(x[a][j]);
        else v[j] = __uint_as_float(j & 1 ? x[a][j >> 1] & 0xFFFF0000u : x[a][j >> 1] << 16);
      }
      uint32_t top = max(max(magnitude(v[0]), magnitude(v[1])), max(magnitude(v[2]), magnitude(v[3])));
      top = max(top, __shfl_xor_sync(four, top, 1));
      top = max(top, __shfl_xor_sync(four, top, 2));
      if (i0 + a * step >= p.total) continue;
      const BlockScale s = block_scale(top);
      uint32_t w;
      block_multiples<4>(v, s.inv, &w);
      int8_t* q = p.c.data + at[a].g * p.c.group + at[a].r * p.c.row + at[a].b * B + c;
      if (left[a] == 4 && ((uint64_t)q & 3) == 0) {
        *reinterpret_cast<uint32_t*>(q) = w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left[a]) q[j] = (int8_t)(w >> 8 * j);
      }
      if (c == 0) p.c.scale[at[a].g * p.c.scale_group + at[a].r * p.c.scale_row + at[a].b] = (uint8_t)s.byte;
    }
  }
}

// And back: a lane takes 16 bytes of y from such a boundary on (a row's first and last in part); their columns are of
// two blocks at most. (p.blocks: units that a row touches at most)
constexpr int UNITS_AHEAD = 4;

template <typename T>
__global__ void __launch_bounds__(256) k_restore_units(const BlocksArgs p) {
  constexpr int E = 16 / sizeof(T);
  pdl_wait();
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < p.total; i0 += UNITS_AHEAD * step) {
    uint32_t q[UNITS_AHEAD][E / 4], byte[UNITS_AHEAD][2];
    T* y[UNITS_AHEAD];
    int64_t col[UNITS_AHEAD];
#pragma unroll
    for (int a = 0; a < UNITS_AHEAD; ++a) {
      col[a] = p.dim;
      if (i0 + a * step >= p.total) continue;
      const At at = block_at(p, i0 + a * step);
      T* row = (T*)p.m.data + at.g * p.m.group + at.r * p.m.row;
      const int64_t c = at.b * E - (int)((uint64_t)row & 15) / (int)sizeof(T);
      if (c >= p.dim) continue;
      col[a] = c, y[a] = row + c;
      const uint8_t* src = (const uint8_t*)p.c.data + at.g * p.c.group + at.r * p.c.row;
      const uint8_t* scale = p.c.scale + at.g * p.c.scale_group + at.r * p.c.scale_row;
      byte[a][0] = __ldg(scale + max(c, (int64_t)0) / B);
      byte[a][1] = __ldg(scale + (min(c + E, p.dim) - 1) / B);
      if (c >= 0 && c + E <= p.dim) {
        const uint4 w = bytes16(src + c, E);
        q[a][0] = w.x;
        if constexpr (E == 8) q[a][1] = w.y;
      } else {
#pragma unroll
        for (int j = 0; j < E / 4; ++j) q[a][j] = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c + e >= 0 && c + e < p.dim) q[a][e / 4] |= (uint32_t)__ldg(src + c + e) << e % 4 * 8;
      }
    }
#pragma unroll
    for (int a = 0; a < UNITS_AHEAD; ++a) {
      if (col[a] >= p.dim) continue;
      const float unit0 = block_unit(byte[a][0]), unit1 = block_unit(byte[a][1]);
      const int border = B - (int)(max(col[a], (int64_t)0) & (B - 1)) + (col[a] < 0 ? (int)-col[a] : 0);
      float v[E];
#pragma unroll
      for (int j = 0; j < E / 4; ++j) block_values(q[a][j], 1.f, v + 4 * j);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= e < border ? unit0 : unit1;
      with_act(p.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < E; e += 2) act_pair<decltype(act)::value, sizeof(T) == 4>(v[e], v[e + 1], p.slope);
      });
      if (col[a] >= 0 && col[a] + E <= p.dim) {
        store_vec<T, E>(y[a], v);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (col[a] + e >= 0 && col[a] + e < p.dim) y[a][e] = from_f<T>(v[e]);
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
dim3 grid_of(const BlocksArgs& p, int per_block) {
  const int64_t want = ceil_div(p.total, per_block), most = 8 * (int64_t)sm_count();
  return dim3((unsigned)(want < most ? want : most));
}

}  // namespace

cudaError_t checkpoint_rows(const lipz_checkpoint_rows_args& a, cudaStream_t st) {
  const BlocksArgs p = blocks_args(a.x, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  const bool fp32 = a.x.type == LIPZ_FP32;
  if (a.dim % (16 / type_bytes(a.x.type)) || !starts_on(p, a.groups, a.rows, 16))
    return fp32 ? launch_pdl(k_checkpoint_quads<float>, grid_of(p, 64), dim3(256), 0, st, p)
                : launch_pdl(k_checkpoint_quads<bf16>, grid_of(p, 64), dim3(256), 0, st, p);
  const bool wide = starts_on(p, a.groups, a.rows, 32);
  if (fp32)
    return wide ? launch_pdl(k_checkpoint<float, true>, grid_of(p, 256), dim3(256), 0, st, p)
                : launch_pdl(k_checkpoint<float, false>, grid_of(p, 256), dim3(256), 0, st, p);
  return wide ? launch_pdl(k_checkpoint<bf16, true>, grid_of(p, 256), dim3(256), 0, st, p)
              : launch_pdl(k_checkpoint<bf16, false>, grid_of(p, 256), dim3(256), 0, st, p);
}

cudaError_t restore_rows(const lipz_restore_rows_args& a, cudaStream_t st) {
  BlocksArgs p = blocks_args(a.y, a.c, a.groups, a.rows, a.dim);
  if (p.total == 0) return cudaSuccess;
  p.act = a.act, p.slope = a.slope;
  const bool fp32 = a.y.type == LIPZ_FP32;
  const int e = 16 / type_bytes(a.y.type);
  if (a.dim % e || !starts_on(p, a.groups, a.rows, 16)) {
    share_out(&p, p.dim == a.dim ? a.groups : 1, ceil_div(p.dim + e - 1, e));
    return fp32 ? launch_pdl(k_restore_units<float>, grid_of(p, 256), dim3(256), 0, st, p)
                : launch_pdl(k_restore_units<bf16>, grid_of(p, 256), dim3(256), 0, st, p);
  }
  const bool wide = starts_on(p, a.groups, a.rows, 32);
  if (fp32)
    return wide ? launch_pdl(k_restore<float, true>, grid_of(p, 256), dim3(256), 0, st, p)
                : launch_pdl(k_restore<float, false>, grid_of(p, 256), dim3(256), 0, st, p);
  return wide ? launch_pdl(k_restore<bf16, true>, grid_of(p, 256), dim3(256), 0, st, p)
              : launch_pdl(k_restore<bf16, false>, grid_of(p, 256), dim3(256), 0, st, p);
}

}  // namespace ops
}  // namespace lipz
