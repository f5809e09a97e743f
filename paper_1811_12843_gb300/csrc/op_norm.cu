// Root-mean-square norm with the residual's addition (forward and backward) and the row quantiser.
//
// A row's elements are read once and stay in the registers of its threads (multiples of 32 of them, NV
// vectors of E elements each) between the row's sums and its results.
// Bound: HBM; a launch and two memory latencies for a few rows.
#include "ops.cuh"

namespace lipz {
namespace ops {

namespace {

struct RowArgs {
  lipz_mat x, residual, sum, y;
  lipz_vec weight, scale, rstd;
  int64_t rows, total;  // of a group, of all
  int dim, tpr, rpb;    // threads per row, rows per block
  float eps;
};

// Sum of a and NaN-propagating maximum of b over the tpr threads of this thread's row. Every thread of
// the block calls it.
__device__ __forceinline__ float2 row_reduce(float a, float b, int tpr, float2* s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b = max_nan(b, __shfl_xor_sync(0xffffffffu, b, o));
  }
  if (tpr > 32) {
    const int warp = threadIdx.x >> 5, w = tpr >> 5, first = threadIdx.x / tpr * w;
    if ((threadIdx.x & 31) == 0) s[warp] = make_float2(a, b);
    __syncthreads();
    float2 r = s[first];
    for (int i = 1; i < w; ++i) {
      const float2 q = s[first + i];
      r.x += q.x;
      r.y = max_nan(r.y, q.y);
    }
    __syncthreads();
    return r;
  }
  return make_float2(a, b);
}

template <typename T>
__device__ __forceinline__ T* row_of(const lipz_mat& m, int64_t g, int64_t r) {
  return reinterpret_cast<T*>(m.data) + g * m.group + r * m.row;
}

// The norm, or with QUANT only the rows' values to 8 bits.
template <typename T, int E, int NV, bool QUANT>
__global__ void __launch_bounds__(E * NV <= 8 ? 1024 : 512) k_rows(const RowArgs p) {
  __shared__ float2 s_red[32];
  const int sub = threadIdx.x / p.tpr, t = threadIdx.x - sub * p.tpr;
  const int64_t r = (int64_t)blockIdx.x * p.rpb + sub;
  const bool live = r < p.total;
  const int64_t g = live ? r / p.rows : 0, gr = live ? r - g * p.rows : 0;
  const int nvec = live ? p.dim / E : 0;
  pdl_wait();
  float v[NV][E];
  const T* x = row_of<const T>(p.x, g, gr);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.tpr;
    if (c < nvec) {
      load_vec<T, E>(x + c * E, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = 0.f;
    }
  }
  const bool q8 = QUANT || p.scale.data;
  const float* weight = QUANT ? nullptr : p.weight.data + g * p.weight.group;
  float ss = 0.f, top = 0.f;
  if (!QUANT) {
    if (p.residual.data) {
      const T* res = row_of<const T>(p.residual, g, gr);
      float w[NV][E];
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * p.tpr < nvec) load_vec<T, E>(res + (t + i * p.tpr) * E, w[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * p.tpr < nvec)
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] += w[i][e];
    }
    if (p.sum.data) {
      T* s = row_of<T>(p.sum, g, gr);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * p.tpr < nvec) store_vec<T, E>(s + (t + i * p.tpr) * E, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(v[i][e], v[i][e], ss);
    if (!QUANT && t + i * p.tpr < nvec) {
      float w[E];
      load_params<E>(weight + (t + i * p.tpr) * E, w);
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] *= w[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
  }
  const float2 red = row_reduce(ss, top, p.tpr, s_red);
  float f = 1.f;
  if (!QUANT) {
    f = 1.f / sqrtf(red.x / (float)p.dim + p.eps);
    if (live && t == 0 && p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = f;
  }
  if (q8) {
    const float scale = max_nan(red.y * f / E4M3_MAX, SCALE_MIN);
    if (live && t == 0) p.scale.data[g * p.scale.group + gr] = scale;
    const float inv = 1.f / scale;  // (two factors: their product may be infinite)
    e4m3* y = row_of<e4m3>(p.y, g, gr);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * p.tpr < nvec) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = v[i][e] * f * inv;
        store_e4m3<E>(y + (t + i * p.tpr) * E, v[i]);
      }
  } else {
    T* y = row_of<T>(p.y, g, gr);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * p.tpr < nvec) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] *= f;
        store_vec<T, E>(y + (t + i * p.tpr) * E, v[i]);
      }
  }
}

// Rows too long for the registers of 1024 threads are read twice, one block per row.
template <typename T, int E>
__global__ void __launch_bounds__(1024) k_quantize_long(const RowArgs p, int64_t dim) {
  __shared__ float2 s_red[32];
  const int64_t r = blockIdx.x, g = r / p.rows, gr = r - g * p.rows;
  const T* x = row_of<const T>(p.x, g, gr);
  e4m3* y = row_of<e4m3>(p.y, g, gr);
  pdl_wait();
  float top = 0.f, v[E];
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < dim / E; c += 1024) {
    load_vec<T, E>(x + c * E, v);
#pragma unroll
    for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[e]));
  }
  const float scale = max_nan(row_reduce(0.f, top, 1024, s_red).y / E4M3_MAX, SCALE_MIN);
  if (threadIdx.x == 0) p.scale.data[g * p.scale.group + gr] = scale;
  const float f = 1.f / scale;
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < dim / E; c += 1024) {
    load_vec<T, E>(x + c * E, v);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= f;
    store_e4m3<E>(y + c * E, v);
  }
}

struct BackArgs {
  lipz_mat dy, s, dsum, dx;
  lipz_vec weight, rstd, dweight;
  float* part;  // [groups][gridDim.x][dim], or null: the block's sums are the group's
  int64_t rows;
  int dim, tpr, rpb;
};

// A block walks over rows of one group (blockIdx.y); its sums for dweight stay in registers, then those
// of its row threads are added in shared memory.
template <typename T, int E, int NV>
__global__ void __launch_bounds__(512) k_rmsnorm_backward(const BackArgs p) {
  extern __shared__ float s_dw[];  // [rpb][dim] where rpb > 1
  __shared__ float2 s_red[32];
  const int sub = threadIdx.x / p.tpr, t = threadIdx.x - sub * p.tpr;
  const int64_t g = blockIdx.y;
  const int nvec = p.dim / E;
  pdl_wait();
  const float* weight = p.weight.data + g * p.weight.group;
  float dw[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) dw[i][e] = 0.f;
  for (int64_t r0 = (int64_t)blockIdx.x * p.rpb; r0 < p.rows; r0 += (int64_t)gridDim.x * p.rpb) {
    const int64_t r = r0 + sub;
    const bool live = r < p.rows;
    Raw<T, E> dy[NV], s[NV];
    const float rstd = live ? p.rstd.data[g * p.rstd.group + r] : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.tpr;
      if (live && c < nvec) {
        dy[i].load(row_of<const T>(p.dy, g, r) + c * E);
        s[i].load(row_of<const T>(p.s, g, r) + c * E);
      } else {
        dy[i].zero();
        s[i].zero();
      }
    }
    float along = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.tpr;
      if (c < nvec) {
        float w[E];
        load_params<E>(weight + c * E, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float ds = dy[i].get(e) * s[i].get(e);
          dw[i][e] = fmaf(ds, rstd, dw[i][e]);
          along = fmaf(ds, w[e], along);
        }
      }
    }
    along = row_reduce(along, 0.f, p.tpr, s_red).x;
    const float c2 = rstd * rstd * (along / (float)p.dim);
    if (live) {
      T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = t + i * p.tpr;
        if (c < nvec) {
          float v[E], w[E];
          load_params<E>(weight + c * E, w);
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] = rstd * fmaf(-s[i].get(e), c2, dy[i].get(e) * w[e]);
          if (p.dsum.data) {
            float d[E];
            load_vec<T, E>(row_of<const T>(p.dsum, g, r) + c * E, d);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += d[e];
          }
          store_vec<T, E>(dx + c * E, v);
        }
      }
    }
  }
  if (!p.dweight.data) return;
  float* out = p.part ? p.part + (g * gridDim.x + blockIdx.x) * (int64_t)p.dim
                      : p.dweight.data + g * p.dweight.group;
  if (p.rpb == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * p.tpr < nvec)
#pragma unroll
        for (int e = 0; e < E; ++e) out[(t + i * p.tpr) * E + e] = dw[i][e];
    return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (t + i * p.tpr < nvec)
#pragma unroll
      for (int e = 0; e < E; ++e) s_dw[sub * p.dim + (t + i * p.tpr) * E + e] = dw[i][e];
  __syncthreads();
  for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
    float v = 0.f;
    for (int q = 0; q < p.rpb; ++q) v += s_dw[q * p.dim + c];
    out[c] = v;
  }
}

// 32 columns by 32 parts per block: each thread adds every 32nd part, then the 32 sums are added.
__global__ void __launch_bounds__(1024)
    k_sum_parts(const float* __restrict__ part, int parts, int64_t cols, lipz_vec out) {
  __shared__ float s[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + tx, g = blockIdx.y;
  pdl_wait();
  float v = 0.f;
  if (c < cols) {
    const float* p = part + g * parts * cols + c;
#pragma unroll 4
    for (int i = ty; i < parts; i += 32) v += p[i * cols];
  }
  s[ty][tx] = v;
  __syncthreads();
  v = s[tx][ty];
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int64_t co = (int64_t)blockIdx.x * 32 + ty;
  if (tx == 0 && co < cols) out.data[g * out.group + co] = v;
}

// Threads per row and vectors per thread: 32 elements per thread reach LIPZ_NORM_MAX_DIM with 512
// threads.
struct RowShape {
  int tpr, nv;
};
int row_threads(int nvec, int nv) { return (int)(ceil_div(ceil_div(nvec, nv), 32) * 32); }
// Few rows: as many threads as vectors (of 4 single elements), so that a row takes one load latency;
// else two vectors per thread, and more where 512 threads of two do not reach the row's end.
template <int E>
RowShape row_shape(int64_t total, int nvec) {
  constexpr int few = E == 1 ? 4 : 1, mid = E == 1 ? 8 : 2;
  if (total <= 2 * sm_count() && row_threads(nvec, few) <= 1024) return {row_threads(nvec, few), few};
  if (row_threads(nvec, mid) <= 512) return {row_threads(nvec, mid), mid};
  return {row_threads(nvec, 32 / E), 32 / E};
}

template <typename T, int E, bool QUANT>
cudaError_t launch_rows(RowArgs& p, cudaStream_t st) {
  constexpr int few = E == 1 ? 4 : 1, mid = E == 1 ? 8 : 2;
  const RowShape s = row_shape<E>(p.total, p.dim / E);
  p.tpr = s.tpr;
  p.rpb = s.tpr >= 256 ? 1 : 256 / s.tpr;
  const dim3 grid((unsigned)ceil_div(p.total, p.rpb)), block(p.tpr * p.rpb);
  if (s.nv == few) return launch_pdl(k_rows<T, E, few, QUANT>, grid, block, 0, st, p);
  if (s.nv == mid) return launch_pdl(k_rows<T, E, mid, QUANT>, grid, block, 0, st, p);
  return launch_pdl(k_rows<T, E, 32 / E, QUANT>, grid, block, 0, st, p);
}

// Vector elements of a backward call: 16 bytes where every row allows it.
bool backward_vec(const lipz_rmsnorm_backward_args& a) {
  const int e = 16 / type_bytes(a.dy.type);
  auto ok = [&](const lipz_mat& m) { return !m.data || rows_aligned(m, a.groups, a.rows, 16); };
  return a.dim % e == 0 && ok(a.dy) && ok(a.s) && ok(a.dsum) && ok(a.dx) &&
         rows_aligned(a.weight, a.groups, 16);
}

struct BackShape {
  RowShape s;
  int rpb, blocks;
};
BackShape backward_shape(const lipz_rmsnorm_backward_args& a) {
  const int e = backward_vec(a) ? 16 / type_bytes(a.dy.type) : 1;
  const int nvec = (int)(a.dim / e);
  const int mid = e == 1 ? 8 : 2;
  BackShape b;
  b.s = row_threads(nvec, mid) <= 256 ? RowShape{row_threads(nvec, mid), mid}
                                      : RowShape{row_threads(nvec, 32 / e), 32 / e};
  b.rpb = b.s.tpr >= 256 ? 1 : 256 / b.s.tpr;
  while (b.rpb > 1 && (int64_t)b.rpb * a.dim * 4 > 48 * 1024) --b.rpb;
  const int64_t fill = 4 * sm_count() * 256 / (b.s.tpr * b.rpb > 256 ? b.s.tpr * b.rpb : 256);
  const int64_t want = fill / (a.groups > 0 ? a.groups : 1);
  const int64_t most = ceil_div(a.rows, b.rpb);
  b.blocks = (int)(want < 1 ? 1 : want > most ? most : want);
  if (b.blocks < 1) b.blocks = 1;
  return b;
}

template <typename T, int E, int NV>
cudaError_t launch_back(const BackArgs& p, int64_t groups, int blocks, cudaStream_t st) {
  return launch_pdl(k_rmsnorm_backward<T, E, NV>, dim3(blocks, (unsigned)groups),
                    dim3(p.tpr * p.rpb), p.rpb > 1 ? (size_t)p.rpb * p.dim * 4 : 0, st, p);
}

template <typename T>
cudaError_t back_type(const BackArgs& p, bool vec, int nv, int64_t groups, int blocks,
                      cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  if (vec) {
    if (nv == 2) return launch_back<T, E, 2>(p, groups, blocks, st);
    return launch_back<T, E, 32 / E>(p, groups, blocks, st);
  }
  if (nv == 8) return launch_back<T, 1, 8>(p, groups, blocks, st);
  return launch_back<T, 1, 32>(p, groups, blocks, st);
}

}  // namespace

cudaError_t rmsnorm(const lipz_rmsnorm_args& a, cudaStream_t st) {
  RowArgs p{a.x, a.residual, a.sum, a.y, a.weight, a.scale, a.rstd, a.rows, a.groups * a.rows,
            (int)a.dim, 0, 0, a.eps};
  if (a.y.type != LIPZ_E4M3) p.scale.data = nullptr;
  if (p.total == 0) return cudaSuccess;
  const int e = 16 / type_bytes(a.x.type);
  auto ok = [&](const lipz_mat& m) {
    return !m.data || rows_aligned(m, a.groups, a.rows, e * type_bytes(m.type));
  };
  const bool vec = a.dim % e == 0 && ok(a.x) && ok(a.residual) && ok(a.sum) && ok(a.y) &&
                   rows_aligned(a.weight, a.groups, 16);
  if (a.x.type == LIPZ_FP32)
    return vec ? launch_rows<float, 4, false>(p, st) : launch_rows<float, 1, false>(p, st);
  return vec ? launch_rows<bf16, 8, false>(p, st) : launch_rows<bf16, 1, false>(p, st);
}

cudaError_t quantize_rows(const lipz_quantize_rows_args& a, cudaStream_t st) {
  RowArgs p{};
  p.x = a.x;
  p.y = a.q;
  p.scale = a.scale;
  p.rows = a.rows;
  p.total = a.groups * a.rows;
  if (p.total == 0) return cudaSuccess;
  const int e = 16 / type_bytes(a.x.type);
  const bool vec = a.dim % e == 0 && rows_aligned(a.x, a.groups, a.rows, 16) &&
                   rows_aligned(a.q, a.groups, a.rows, e);
  if (a.dim > LIPZ_NORM_MAX_DIM) {
    p.tpr = 1024;
    const dim3 grid((unsigned)p.total), block(1024);
    if (a.x.type == LIPZ_FP32)
      return vec ? launch_pdl(k_quantize_long<float, 4>, grid, block, 0, st, p, a.dim)
                 : launch_pdl(k_quantize_long<float, 1>, grid, block, 0, st, p, a.dim);
    return vec ? launch_pdl(k_quantize_long<bf16, 8>, grid, block, 0, st, p, a.dim)
               : launch_pdl(k_quantize_long<bf16, 1>, grid, block, 0, st, p, a.dim);
  }
  p.dim = (int)a.dim;
  if (a.x.type == LIPZ_FP32)
    return vec ? launch_rows<float, 4, true>(p, st) : launch_rows<float, 1, true>(p, st);
  return vec ? launch_rows<bf16, 8, true>(p, st) : launch_rows<bf16, 1, true>(p, st);
}

cudaError_t sum_parts(const float* part, int64_t groups, int parts, int64_t cols, lipz_vec out,
                      cudaStream_t st) {
  return launch_pdl(k_sum_parts, dim3((unsigned)ceil_div(cols, 32), (unsigned)groups), dim3(1024), 0,
                    st, part, parts, cols, out);
}

int rmsnorm_backward_blocks(const lipz_rmsnorm_backward_args& a) { return backward_shape(a).blocks; }

cudaError_t rmsnorm_backward(const lipz_rmsnorm_backward_args& a, cudaStream_t st) {
  if (a.groups == 0) return cudaSuccess;
  const BackShape b = backward_shape(a);
  BackArgs p{a.dy, a.s, a.dsum, a.dx, a.weight, a.rstd, a.dweight, nullptr, a.rows, (int)a.dim,
             b.s.tpr, b.rpb};
  if (b.blocks > 1) p.part = (float*)a.workspace;
  const bool vec = backward_vec(a);
  cudaError_t e = a.dy.type == LIPZ_FP32 ? back_type<float>(p, vec, b.s.nv, a.groups, b.blocks, st)
                                         : back_type<bf16>(p, vec, b.s.nv, a.groups, b.blocks, st);
  if (e != cudaSuccess || b.blocks == 1 || !a.dweight.data) return e;
  return sum_parts(p.part, a.groups, b.blocks, a.dim, a.dweight, st);
}

}  // namespace ops
}  // namespace lipz
