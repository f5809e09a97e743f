// Layer norm with the residual's addition, forward (with the sum kept in 8 bits) and backward.
//
// A row's elements are read once and stay in the registers of its threads (multiples of 32 of them, NV
// vectors of E elements each) between the row's sums and its results. Bound: HBM; a launch and two memory
// latencies for a few rows.
#include "op_rows.cuh"

namespace lipz {
namespace ops {

namespace {

struct LayerArgs {
  lipz_mat x, residual, sum, y;
  lipz_vec weight, bias, scale, mean, rstd;
  lipz_blocks kept;
  int64_t rows, total;  // of a group, of all
  int dim, tpr, rpb;    // threads per row, rows per block
  float eps, inv_dim;
};

// (rows of all groups stay below 2^31)
__device__ __forceinline__ int64_t group_at(int64_t r, int64_t rows, int64_t total) {
  return total == rows ? 0 : (uint32_t)r / (uint32_t)rows;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A warp's share of a row: how many elements, their sum, and the sum of the squares of their distances from their
// own mean. Shares are joined without a difference of near values:
//     mean = sum of sums / n;  sum (v - mean)^2 = sum over shares of (m2 + n_i (mean_i - mean)^2)
struct Share {
  float n, sum, m2;
};
struct Moments {
  float mean, rstd;
};
__device__ __forceinline__ Moments join_shares(const Share* s, int warps, float inv_dim, float eps) {
  float sum = 0.f, m2 = 0.f;
  for (int i = 0; i < warps; ++i) sum += s[i].sum;
  const float mean = sum * inv_dim;
  for (int i = 0; i < warps; ++i)
    if (s[i].n > 0.f) {
      const float off = s[i].sum / s[i].n - mean;
      m2 += fmaf(s[i].n * off, off, s[i].m2);
    }
  return {mean, rsqrtf(fmaf(m2, inv_dim, eps))};
}

// E elements of a row, as they are written to sum (rounded to T), to its checkpoint: 16 / E lanes hold a block, and
// all of a warp's lanes call it (live: this lane's elements are part of the row).
template <typename T, int E>
__device__ __forceinline__ void keep_vec(int8_t* q, uint8_t* scale, int col, bool live, const float* v) {
  float u[E];
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    u[e] = to_f<T>(from_f<T>(v[e]));
    if (live) top = max(top, magnitude(u[e]));
  }
#pragma unroll
  for (int o = 1; o < LIPZ_BLOCK / E; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!live) return;
  const BlockScale s = block_scale(top);
  if constexpr (E == 1) {
    q[col] = (int8_t)block_multiple(u[0], s.inv);
  } else {
    uint32_t w[E / 4];
    block_multiples<E>(u, s.inv, w);
    if constexpr (E == 8) *reinterpret_cast<uint2*>(q + col) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q + col) = w[0];
  }
  if (col % LIPZ_BLOCK == 0) scale[col / LIPZ_BLOCK] = (uint8_t)s.byte;
}

template <typename T, int E, int NV>
__global__ void __launch_bounds__(E * NV <= 8 ? 1024 : 512) k_layer_rows(const LayerArgs p) {
  __shared__ Share s_share[32];
  __shared__ uint32_t s_top[32];
  const int sub = threadIdx.x / p.tpr, t = threadIdx.x - sub * p.tpr, warps = p.tpr >> 5;
  const int64_t r = (int64_t)blockIdx.x * p.rpb + sub;
  const bool live = r < p.total;
  const int64_t g = live ? group_at(r, p.rows, p.total) : 0, gr = live ? r - g * p.rows : 0;
  const int nvec = live ? p.dim / E : 0;
  pdl_wait();
  float v[NV][E];
  const T* x = row_of<const T>(p.x, g, gr);
  int held = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.tpr;
    if (c < nvec) {
      load_vec<T, E>(x + c * E, v[i]);
      held += E;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = 0.f;
    }
  }
  if (p.residual.data) {
    const T* res = row_of<const T>(p.residual, g, gr);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * p.tpr < nvec) {
        float w[E];
        load_vec<T, E>(res + (t + i * p.tpr) * E, w);
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] += w[e];
      }
  }
  if (p.sum.data) {
    T* s = row_of<T>(p.sum, g, gr);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * p.tpr < nvec) store_vec<T, E>(s + (t + i * p.tpr) * E, v[i]);
  }
  if (p.kept.data) {
    int8_t* q = p.kept.data + g * p.kept.group + gr * p.kept.row;
    uint8_t* scale = p.kept.scale + g * p.kept.scale_group + gr * p.kept.scale_row;
#pragma unroll
    for (int i = 0; i < NV; ++i) keep_vec<T, E>(q, scale, (t + i * p.tpr) * E, t + i * p.tpr < nvec, v[i]);
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) sum += v[i][e];
  sum = warp_sum(sum);
  const float n = (float)__reduce_add_sync(0xffffffffu, held), own = n > 0.f ? sum / n : 0.f;
  float m2 = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (t + i * p.tpr < nvec)
#pragma unroll
      for (int e = 0; e < E; ++e) m2 = fmaf(v[i][e] - own, v[i][e] - own, m2);
  m2 = warp_sum(m2);
  const int warp = threadIdx.x >> 5, first = sub * warps;
  if ((threadIdx.x & 31) == 0) s_share[warp] = {n, sum, m2};
  __syncthreads();
  const Moments mo = join_shares(s_share + first, warps, p.inv_dim, p.eps);
  const float* weight = p.weight.data + g * p.weight.group;
  const float* bias = p.bias.data ? p.bias.data + g * p.bias.group : nullptr;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.tpr;
    if (c >= nvec) continue;
    float w[E], b[E];
    load_params<E>(weight + c * E, w);
#pragma unroll
    for (int e = 0; e < E; ++e) b[e] = 0.f;
    if (bias) load_params<E>(bias + c * E, b);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[i][e] = fmaf((v[i][e] - mo.mean) * mo.rstd, w[e], b[e]);
      top = max(top, magnitude(v[i][e]));
    }
  }
  Reciprocal inv{1.f, 0.f};
  if (p.scale.data) {
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) s_top[warp] = top;
    __syncthreads();
    for (int i = 0; i < warps; ++i) top = max(top, s_top[first + i]);
    const float scale = scale_of(__uint_as_float(top));
    inv = reciprocal_of(scale);
    if (live && t == 0) p.scale.data[g * p.scale.group + gr] = scale;
  }
  if (!live) return;
  if (t == 0) {
    if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
    if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.tpr;
    if (c >= nvec) continue;
    if (p.scale.data) {
      scale_by<E>(v[i], inv);
      store_e4m3<E>(row_of<e4m3>(p.y, g, gr) + c * E, v[i]);
    } else {
      store_vec<T, E>(row_of<T>(p.y, g, gr) + c * E, v[i]);
    }
  }
}

template <typename T, int E>
cudaError_t launch_layer(LayerArgs& p, cudaStream_t st) {
  // as many threads as vectors (of 4 single elements), so that a row takes one load latency
  constexpr int few = E == 1 ? 4 : 1;
  const int nvec = p.dim / E, nv = row_threads(nvec, few) <= 1024 ? few : 32 / E;
  p.tpr = row_threads(nvec, nv);
  p.rpb = p.tpr >= 256 ? 1 : 256 / p.tpr;
  const dim3 grid((unsigned)ceil_div(p.total, p.rpb)), block(p.tpr * p.rpb);
  return nv == few ? launch_pdl(k_layer_rows<T, E, few>, grid, block, 0, st, p)
                   : launch_pdl(k_layer_rows<T, E, 32 / E>, grid, block, 0, st, p);
}

// ---- backward

struct LayerBack {
  lipz_mat dy, s, dsum, dx;
  lipz_blocks kept;
  lipz_vec weight, mean, rstd, dweight, dbias;
  float* part;  // [groups][blocks][2][dim]: sums for dweight and dbias, or null: those of one are the group's
  int64_t rows;
  int dim;
  float inv_dim;
};

// A block of one row's threads walks over rows of one group (blockIdx.y); the sums over its rows stay in registers.
template <typename T, int E, int NV, bool KEPT>
__global__ void __launch_bounds__(512) k_layer_backward(const LayerBack p) {
  __shared__ float2 s_red[2][16];
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, tpr = blockDim.x, nvec = p.dim / E, warps = tpr >> 5;
  pdl_wait();
  const float* weight = p.weight.data + g * p.weight.group;
  float dw[NV][E], db[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) dw[i][e] = db[i][e] = 0.f;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn ^= 1) {
    const float mean = p.mean.data[g * p.mean.group + r], rstd = p.rstd.data[g * p.rstd.group + r];
    float dy[NV][E], s[NV][E];
    float2 sums = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      if (c >= nvec) continue;
      load_vec<T, E>(row_of<const T>(p.dy, g, r) + c * E, dy[i]);
      if constexpr (KEPT) {
        const int8_t* q = p.kept.data + g * p.kept.group + r * p.kept.row + c * E;
        const float unit = block_unit(
            p.kept.scale[g * p.kept.scale_group + r * p.kept.scale_row + c * E / LIPZ_BLOCK]);
        if constexpr (E == 1) {
          s[i][0] = (float)*q * unit;
        } else {
#pragma unroll
          for (int e = 0; e < E; e += 4) block_values(*reinterpret_cast<const uint32_t*>(q + e), unit, s[i] + e);
        }
      } else {
        load_vec<T, E>(row_of<const T>(p.s, g, r) + c * E, s[i]);
      }
      float w[E];
      load_params<E>(weight + c * E, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s[i][e] -= mean;
        const float m = dy[i][e] * s[i][e];
        dw[i][e] = fmaf(m, rstd, dw[i][e]);
        db[i][e] += dy[i][e];
        sums.x = fmaf(dy[i][e], w[e], sums.x);
        sums.y = fmaf(m, w[e], sums.y);
      }
    }
    sums.x = warp_sum(sums.x), sums.y = warp_sum(sums.y);
    if ((t & 31) == 0) s_red[turn][t >> 5] = sums;
    __syncthreads();
    sums = s_red[turn][0];
    for (int i = 1; i < warps; ++i) sums.x += s_red[turn][i].x, sums.y += s_red[turn][i].y;
    // (rstd^2 by itself may be infinite where the gradient is not)
    const float c1 = sums.x * p.inv_dim, c2 = rstd * (rstd * (sums.y * p.inv_dim));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      if (c >= nvec) continue;
      float w[E], ds[E];
      load_params<E>(weight + c * E, w);
#pragma unroll
      for (int e = 0; e < E; ++e) ds[e] = 0.f;
      if (p.dsum.data) load_vec<T, E>(row_of<const T>(p.dsum, g, r) + c * E, ds);
#pragma unroll
      for (int e = 0; e < E; ++e)
        ds[e] = fmaf(rstd, fmaf(-s[i][e], c2, fmaf(dy[i][e], w[e], -c1)), ds[e]);
      store_vec<T, E>(row_of<T>(p.dx, g, r) + c * E, ds);
    }
  }
  float* out[2] = {p.dweight.data ? p.dweight.data + g * p.dweight.group : nullptr,
                   p.dbias.data ? p.dbias.data + g * p.dbias.group : nullptr};
  if (p.part) out[0] = p.part + (g * gridDim.x + blockIdx.x) * 2 * p.dim, out[1] = out[0] + p.dim;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (t + i * tpr < nvec)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (t + i * tpr) * E + e;
        if (out[0]) out[0][c] = dw[i][e];
        if (out[1]) out[1][c] = db[i][e];
      }
}

// 32 columns per block, blockDim.y parts at a time, of dweight's sums (blockIdx.z = 0) or dbias's.
__global__ void __launch_bounds__(1024)
    k_sum_pairs(const float* __restrict__ part, int parts, int64_t cols, lipz_vec dweight, lipz_vec dbias) {
  __shared__ float s[32][33];
  const lipz_vec out = blockIdx.z ? dbias : dweight;
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x, g = blockIdx.y;
  pdl_wait();
  if (!out.data) return;
  float v = 0.f;
  if (c < cols) {
    const float* p = part + (g * parts * 2 + blockIdx.z) * cols + c;
    for (int i0 = threadIdx.y; i0 < parts; i0 += 16 * blockDim.y) {
      float w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int i = i0 + j * blockDim.y;
        w[j] = i < parts ? __ldg(p + i * 2 * cols) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) v += w[j];
    }
  }
  s[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.y || c >= cols) return;
  for (int i = 1; i < blockDim.y; ++i) v += s[i][threadIdx.x];
  out.data[g * out.group + c] = v;
}

// Vector elements of a backward call: 16 bytes where every row allows it.
bool back_vec(const lipz_layernorm_backward_args& a) {
  const int e = 16 / type_bytes(a.dy.type);
  auto ok = [&](const lipz_mat& m) { return !m.data || rows_aligned(m, a.groups, a.rows, 16); };
  return a.dim % e == 0 && ok(a.dy) && ok(a.dsum) && ok(a.dx) &&
         (a.kept.data ? rows_aligned(bytes_of(a.kept), a.groups, a.rows, e) : ok(a.s)) &&
         rows_aligned(a.weight, a.groups, 16);
}

int back_blocks(const lipz_layernorm_backward_args& a) {
  const int64_t groups = a.groups > 0 ? a.groups : 1;
  const int64_t fill = ceil_div(2 * (int64_t)sm_count(), groups), most = ceil_div(a.rows, 4);
  const int64_t b = fill < most ? fill : most;
  return b < 1 ? 1 : (int)b;
}

template <typename T, int E, bool KEPT>
cudaError_t launch_layer_back(const LayerBack& p, int64_t groups, int blocks, cudaStream_t st) {
  const int nvec = p.dim / E, nv = row_threads(nvec, 16 / E) <= 512 ? 16 / E : 32 / E;
  const dim3 grid(blocks, (unsigned)groups), block(row_threads(nvec, nv));
  return nv == 16 / E ? launch_pdl(k_layer_backward<T, E, 16 / E, KEPT>, grid, block, 0, st, p)
                      : launch_pdl(k_layer_backward<T, E, 32 / E, KEPT>, grid, block, 0, st, p);
}
template <typename T, bool KEPT>
cudaError_t launch_layer_back(const LayerBack& p, bool vec, int64_t groups, int blocks, cudaStream_t st) {
  return vec ? launch_layer_back<T, 16 / sizeof(T), KEPT>(p, groups, blocks, st)
             : launch_layer_back<T, 1, KEPT>(p, groups, blocks, st);
}

}  // namespace

cudaError_t layernorm(const lipz_layernorm_args& a, cudaStream_t st) {
  LayerArgs p{a.x, a.residual, a.sum, a.y, a.weight, a.bias, a.scale, a.mean, a.rstd, a.kept,
              a.rows, a.groups * a.rows, (int)a.dim, 0, 0, a.eps, 1.f / (float)a.dim};
  if (a.y.type != LIPZ_E4M3) p.scale.data = nullptr;
  if (p.total == 0) return cudaSuccess;
  const int e = 16 / type_bytes(a.x.type);
  auto ok = [&](const lipz_mat& m) {
    return !m.data || rows_aligned(m, a.groups, a.rows, e * type_bytes(m.type));
  };
  const bool vec = a.dim % e == 0 && ok(a.x) && ok(a.residual) && ok(a.sum) && ok(a.y) && ok(bytes_of(a.kept)) &&
                   rows_aligned(a.weight, a.groups, 16) && (!a.bias.data || rows_aligned(a.bias, a.groups, 16));
  if (a.x.type == LIPZ_FP32) return vec ? launch_layer<float, 4>(p, st) : launch_layer<float, 1>(p, st);
  return vec ? launch_layer<bf16, 8>(p, st) : launch_layer<bf16, 1>(p, st);
}

uint64_t layernorm_backward_workspace(const lipz_layernorm_backward_args& a) {
  const int blocks = back_blocks(a);
  return (a.dweight.data || a.dbias.data) && blocks > 1 ? (uint64_t)a.groups * blocks * 2 * a.dim * 4 : 0;
}

cudaError_t layernorm_backward(const lipz_layernorm_backward_args& a, cudaStream_t st) {
  if (a.groups == 0) return cudaSuccess;
  const int blocks = back_blocks(a);
  const bool parts = blocks > 1 && (a.dweight.data || a.dbias.data);
  const LayerBack p{a.dy, a.s, a.dsum, a.dx, a.kept, a.weight, a.mean, a.rstd, a.dweight, a.dbias,
                    parts ? (float*)a.workspace : nullptr, a.rows, (int)a.dim, 1.f / (float)a.dim};
  const bool vec = back_vec(a), kept = a.kept.data;
  cudaError_t e;
  if (a.dy.type == LIPZ_FP32)
    e = kept ? launch_layer_back<float, true>(p, vec, a.groups, blocks, st)
             : launch_layer_back<float, false>(p, vec, a.groups, blocks, st);
  else
    e = kept ? launch_layer_back<bf16, true>(p, vec, a.groups, blocks, st)
             : launch_layer_back<bf16, false>(p, vec, a.groups, blocks, st);
  if (e != cudaSuccess || !parts) return e;
  const int ways = blocks >= 128 ? 32 : blocks >= 16 ? 8 : 1;
  return launch_pdl(k_sum_pairs, dim3((unsigned)ceil_div(a.dim, 32), (unsigned)a.groups, 2), dim3(32, ways), 0, st,
                    p.part, blocks, (int64_t)a.dim, a.dweight, a.dbias);
}

}  // namespace ops
}  // namespace lipz
