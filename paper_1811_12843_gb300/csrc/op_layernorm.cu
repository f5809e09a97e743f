// Layer norm with the residual's addition, forward (with the sum kept in 8 bits) and backward.
//
//     s = x + residual,  y = (s - mean) rstd w + b,  rstd = 1 / sqrt(mean((s - mean)^2) + eps)
//     g = dy w,  dx = rstd (g - mean(g) - (s - mean) rstd^2 mean(g (s - mean))) + dsum
//     dw = sum over rows of dy (s - mean) rstd,  db = sum over rows of dy
//
// A row's elements are read once and stay in the registers of its threads (multiples of 32 of them, NV
// vectors of E elements each) between the row's sums and its results, all in fp32, in an order that only sizes
// decide. The sum of squares is of distances from means (join_shares), so that a row far from zero loses no more than
// the rounding of its elements and of those means.
//
// Bound: HBM, and what a row's two sums make it wait for; a launch and two memory latencies for a few rows.
// Measured (a copy runs at 6784 GB/s; inputs larger than L2, a call's time among others):
//   to bf16 and a checkpoint, with a residual, 16384 x 8192   204 us  0.88 of the copy rate (k_layer_stream)
//   fp32, 8193 x 1001, with a residual                        27 us   0.72 (k_layer_stream, SHIFT)
//   backward with dsum, 8192 x 4096                           56 us   0.70 (k_layer_back_stream, k_sum_pairs)
//   backward over a checkpoint with dsum, 16384 x 2048        60 us   0.58 (the same)
//   backward with dsum, 144 groups of 100 x 256               8.2 us  latency (k_layer_back_short)
//   one row of 4096 to 8 bits                                 2.9 us  in a graph (k_layer_rows)
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

// Widest rows that are taken in units off the 16-byte grid: 512 threads of 16 elements, less the unit more.
constexpr int SHIFT_DIM = 512 * 16 - 8;

// (rows of all groups stay below 2^31)
__device__ __forceinline__ int64_t group_at(int64_t r, int64_t rows, int64_t total) {
  return total == rows ? 0 : (uint32_t)r / (uint32_t)rows;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A warp's share of a row: how many elements, their sum and mean, and the sum of the squares of their distances from
// that mean (x to w). Shares are joined without a difference of near values:
//     mean = sum of sums / n;  sum (v - mean)^2 = sum over shares of (m2 + n_i (mean_i - mean)^2)
struct Moments {
  float mean, rstd;
};
// (by the lanes of each warp, a share to each, up to 32; every warp has the sums in the same order)
__device__ __forceinline__ Moments join_shares(const float4* s, int warps, float inv_dim, float eps) {
  const int lane = threadIdx.x & 31;
  const float4 q = lane < warps ? s[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = q.y;
  for (int o = 1; o < warps; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const float mean = __shfl_sync(0xffffffffu, sum, 0) * inv_dim, off = q.z - mean;
  float m2 = q.x > 0.f ? fmaf(q.x * off, off, q.w) : 0.f;
  for (int o = 1; o < warps; o <<= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
  m2 = __shfl_sync(0xffffffffu, m2, 0);
  return {mean, rsqrtf(fmaf(m2, inv_dim, eps))};
}

// Sums over a thread's vectors, two elements at a time; count: how many of the NV vectors are part of the row (the
// others hold zeros).
template <int E, int NV>
__device__ __forceinline__ float sum_of(const float (&v)[NV][E]) {
  if constexpr (E == 1) {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) a += v[i][0];
    return a;
  } else {
    uint64_t a = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; e += 2) a = add2(a, pack2(v[i][e], v[i][e + 1]));
    const float2 r = unpack2(a);
    return r.x + r.y;
  }
}
template <int E, int NV>
__device__ __forceinline__ float squares_of(const float (&v)[NV][E], float mean, int count) {
  if constexpr (E == 1) {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) a = fmaf(v[i][0] - mean, v[i][0] - mean, a);
    return a;
  } else {
    uint64_t a = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count)
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const uint64_t d = add2(pack2(v[i][e], v[i][e + 1]), both(-mean));
          a = fma2(d, d, a);
        }
    const float2 r = unpack2(a);
    return r.x + r.y;
  }
}
// v = (v - mean) rstd w + b
template <int E>
__device__ __forceinline__ void affine(float* v, Moments mo, const float* w, const float* b) {
  if constexpr (E == 1) {
    v[0] = fmaf((v[0] - mo.mean) * mo.rstd, w[0], b[0]);
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const uint64_t d = mul2(add2(pack2(v[e], v[e + 1]), both(-mo.mean)), both(mo.rstd));
      const float2 r = unpack2(fma2(d, pack2(w[e], w[e + 1]), pack2(b[e], b[e + 1])));
      v[e] = r.x, v[e + 1] = r.y;
    }
  }
}

// E elements of a row, as they are written to sum (rounded to T), to its checkpoint: 16 / E lanes hold a block, and
// all of a warp's lanes call it (live: this lane's elements are part of the row).
template <typename T, int E>
__device__ __forceinline__ void keep_vec(int8_t* q, uint8_t* scale, int col, bool live, const float* v) {
  float u[E];
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    u[e] = to_f<T>(from_f<T>(v[e]));
    if (live) most = max_nan(most, fabsf(u[e]));
  }
  uint32_t top = __float_as_uint(most);
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

// ---- elements two to a 64-bit register pair, as the instructions over two of them take them. (Arrays of single
// elements cost as many moves as there are operations: 16384 x 8192 with a checkpoint 250 us, so 217.)
template <typename T, int E>
__device__ __forceinline__ void pairs_of(const Raw<T, E>& r, uint64_t* v) {
#pragma unroll
  for (int j = 0; j < E / 2; ++j) v[j] = pack2(r.get(2 * j), r.get(2 * j + 1));
}
// (eight by one access where they lie on 32 bytes: lanes 32 bytes apart meet each line once)
template <int E>
__device__ __forceinline__ void load_pairs(const float* p, uint64_t* w) {
  if constexpr (E == 8) {
    if (((uint64_t)p & 31) == 0) {
      asm("ld.global.nc.v4.b64 {%0,%1,%2,%3}, [%4];" : "=l"(w[0]), "=l"(w[1]), "=l"(w[2]), "=l"(w[3]) : "l"(p));
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < E / 2; j += 2) {
    const ulonglong2 r = __ldg(reinterpret_cast<const ulonglong2*>(p + 2 * j));
    w[j] = r.x, w[j + 1] = r.y;
  }
}
// As they are written: rounded to T.
template <typename T, int E>
__device__ __forceinline__ Raw<T, E> rounded(const uint64_t* v) {
  Raw<T, E> r;
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const float2 f = unpack2(v[j]);
    if constexpr (sizeof(T) == 4) {
      r.w[2 * j] = __float_as_uint(f.x), r.w[2 * j + 1] = __float_as_uint(f.y);
    } else {
      r.w[j] = tc::pack_bf16(f.x, f.y);
    }
  }
  return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_raw(T* p, const Raw<T, E>& r) {
  *reinterpret_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
}
template <typename T, int E>
__device__ __forceinline__ void store_pairs(T* p, const uint64_t* v) {
  store_raw<T, E>(p, rounded<T, E>(v));
}
template <int E>
__device__ __forceinline__ void store_pairs_e4m3(e4m3* p, const uint64_t* v, Reciprocal inv) {
  uint32_t h[E / 2];
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const float2 f = unpack2(fma2(v[j], both(inv.hi), mul2(v[j], both(inv.lo))));
    h[j] = e4m3x2(f.x, f.y);
  }
  if constexpr (E == 8) *reinterpret_cast<uint2*>(p) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
  else *reinterpret_cast<uint32_t*>(p) = h[0] | h[1] << 16;
}
// The largest magnitude's bits of a vector as it is written.
template <typename T, int E>
__device__ __forceinline__ uint32_t top_of(const Raw<T, E>& r) {
  if constexpr (sizeof(T) == 4) {
    float m = fabsf(r.get(0));
#pragma unroll
    for (int e = 1; e < E; ++e) m = max_nan(m, fabsf(r.get(e)));
    return __float_as_uint(m);
  } else {
    uint32_t m = r.w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int j = 1; j < E / 2; ++j)
      asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[j] & 0x7FFF7FFFu));
    return max(m << 16, m & 0xFFFF0000u);
  }
}
// A vector, as it is written to sum, to its checkpoint: 16 / E lanes hold a block, and all of a warp's lanes call it
// (live: this lane's elements are part of the row).
template <typename T, int E>
__device__ __forceinline__ void keep_raw(int8_t* q, uint8_t* scale, int col, bool live, const Raw<T, E>& r) {
  uint32_t top = live ? top_of<T, E>(r) : 0u;
#pragma unroll
  for (int o = 1; o < LIPZ_BLOCK / E; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!live) return;
  const BlockScale s = block_scale(top);
  uint32_t w[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    const float2 a = unpack2(fma2(pack2(r.get(4 * i), r.get(4 * i + 1)), both(s.inv), both(12582912.f)));
    const float2 b = unpack2(fma2(pack2(r.get(4 * i + 2), r.get(4 * i + 3)), both(s.inv), both(12582912.f)));
    w[i] = pack_bytes(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
  if constexpr (E == 8) *reinterpret_cast<uint2*>(q + col) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(q + col) = w[0];
  if (col % LIPZ_BLOCK == 0) scale[col / LIPZ_BLOCK] = (uint8_t)s.byte;
}
template <int N>
__device__ __forceinline__ float pairs_sum(const uint64_t (&v)[N]) {
  uint64_t a = v[0];
#pragma unroll
  for (int j = 1; j < N; ++j) a = add2(a, v[j]);
  const float2 r = unpack2(a);
  return r.x + r.y;
}
// Of the squares of distances from a mean, over the vectors of a set.
template <int E, int NV>
__device__ __forceinline__ float pairs_squares(const uint64_t (&v)[NV * E / 2], float mean, uint32_t set) {
  uint64_t a = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (set >> i & 1)
#pragma unroll
      for (int j = 0; j < E / 2; ++j) {
        const uint64_t d = add2(v[i * (E / 2) + j], both(-mean));
        a = fma2(d, d, a);
      }
  const float2 r = unpack2(a);
  return r.x + r.y;
}
// v = (v - mean) rstd w + b; returns the largest magnitude if it is wanted.
template <int E, bool MAX>
__device__ __forceinline__ float pairs_affine(uint64_t* v, Moments mo, const uint64_t* w, const uint64_t* b, float top) {
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    v[j] = fma2(mul2(add2(v[j], both(-mo.mean)), both(mo.rstd)), w[j], b[j]);
    if constexpr (MAX) {
      const float2 f = unpack2(v[j]);
      top = max_nan(max_nan(top, fabsf(f.x)), fabsf(f.y));
    }
  }
  return top;
}

// Results of a row that is in registers: statistics kept, y or its 8 bits.
template <typename T, int E, int NV>
__device__ __forceinline__ void layer_results(const LayerArgs& p, int64_t g, int64_t gr, Moments mo, Reciprocal inv,
                                              float (&v)[NV][E], int t, int tpr, int nvec) {
  if (t == 0) {
    if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
    if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * tpr;
    if (c >= nvec) continue;
    if (p.scale.data) {
      scale_by<E>(v[i], inv);
      store_e4m3<E>(row_of<e4m3>(p.y, g, gr) + c * E, v[i]);
    } else {
      store_vec<T, E>(row_of<T>(p.y, g, gr) + c * E, v[i]);
    }
  }
}

// Few rows, and rows whose matrices lie at different places of a 16-byte unit: loaded by the threads that use them.
template <typename T, int E, int NV>
__global__ void __launch_bounds__(E * NV <= 8 ? 1024 : 512) k_layer_rows(const LayerArgs p) {
  __shared__ float4 s_share[32];
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
      ++held;
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
  const float sum = warp_sum(sum_of<E, NV>(v));
  const float n = (float)__reduce_add_sync(0xffffffffu, held * E), own = n > 0.f ? sum / n : 0.f;
  const float m2 = warp_sum(squares_of<E, NV>(v, own, held));
  const int warp = threadIdx.x >> 5, first = sub * warps;
  if ((threadIdx.x & 31) == 0) s_share[warp] = make_float4(n, sum, own, m2);
  __syncthreads();
  const Moments mo = join_shares(s_share + first, warps, p.inv_dim, p.eps);
  const float* weight = p.weight.data + g * p.weight.group;
  const float* bias = p.bias.data ? p.bias.data + g * p.bias.group : nullptr;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.tpr;
    if (c >= nvec) continue;
    float w[E], b[E];
    load_params<E>(weight + c * E, w);
#pragma unroll
    for (int e = 0; e < E; ++e) b[e] = 0.f;
    if (bias) load_params<E>(bias + c * E, b);
    affine<E>(v[i], mo, w, b);
#pragma unroll
    for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
  }
  Reciprocal inv{1.f, 0.f};
  if (p.scale.data) {
    uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
    if ((threadIdx.x & 31) == 0) s_top[warp] = most;
    __syncthreads();
    for (int i = 0; i < warps; ++i) most = max(most, s_top[first + i]);
    const float scale = scale_of(__uint_as_float(most));
    inv = reciprocal_of(scale);
    if (live && t == 0) p.scale.data[g * p.scale.group + gr] = scale;
  }
  if (live) layer_results<T, E, NV>(p, g, gr, mo, inv, v, t, p.tpr, nvec);
}

// The units of a row off the 16-byte grid: a thread's columns are c E - m + e, the row's first and last unit in part.
template <int E>
struct Units {
  int m, dim;  // elements of the first unit before the row
  __device__ __forceinline__ int col(int c) const { return c * E - m; }
  __device__ __forceinline__ bool live(int c) const { return c * E - m < dim; }
  __device__ __forceinline__ bool whole(int c) const { return c * E >= m && c * E - m + E <= dim; }
  __device__ __forceinline__ bool in(int c, int e) const { return c * E - m + e >= 0 && c * E - m + e < dim; }
  __device__ __forceinline__ int count(int c) const { return min(c * E - m + E, dim) - max(c * E - m, 0); }
  // a unit's parameters, zeros beside the row
  __device__ __forceinline__ void params(const float* p, int c, uint64_t* w) const {
#pragma unroll
    for (int e = 0; e < E; e += 2)
      w[e / 2] = pack2(in(c, e) ? __ldg(p + col(c) + e) : 0.f, in(c, e + 1) ? __ldg(p + col(c) + e + 1) : 0.f);
  }
};
template <typename T, int E>
__device__ __forceinline__ void store_edge(T* row, const Units<E>& u, int c, const Raw<T, E>& r) {
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (u.in(c, e)) row[u.col(c) + e] = from_f<T>(r.get(e));
}

template <int E>
__device__ __forceinline__ void store_edge_e4m3(e4m3* row, const Units<E>& u, int c, const uint64_t* v, Reciprocal inv) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float2 f = unpack2(v[e / 2]);
    float one = e & 1 ? f.y : f.x;
    scale_by<1>(&one, inv);
    if (u.in(c, e)) store_e4m3<1>(row + u.col(c) + e, &one);
  }
}

// ---- many short rows: a warp walks over sets of 32 / L rows, L lanes to a row of NV vectors each. The next set's
// loads are in flight while this one is summed and written; weights and biases stay in a lane's registers where a
// lane has 16 elements. No barrier.
constexpr int SHORT_WARPS = 4;  // of a block

// SHIFT: rows off the 16-byte grid, which all begin at the same place of a unit for a lane: the rows that it takes lie a
// multiple of 16 rows' bytes apart. (131072 x 77 through rings, a row per warp, 88 us, so 35; 65536 x 301 66 both ways.)
template <typename T, int E, int NV, int L, bool SHIFT>
__global__ void __launch_bounds__(32 * SHORT_WARPS, E == 4 && NV == 8 ? 3 : 4) k_layer_short(const LayerArgs p) {
  constexpr int R = 32 / L, P = E / 2;
  constexpr bool HELD = NV * E <= 16;
  static_assert(!SHIFT || HELD, "parameters in registers");
  const int lane = threadIdx.x & 31, t = lane % L, sub = lane / L;
  const int64_t step = (int64_t)gridDim.x * SHORT_WARPS * R;
  int64_t r = ((int64_t)blockIdx.x * SHORT_WARPS + (threadIdx.x >> 5)) * R + sub;
  const bool has_res = p.residual.data;
  auto group = [&](int64_t at) { return at < p.total ? group_at(at, p.rows, p.total) : 0; };
  const Units<E> units{
      SHIFT ? (int)((uint64_t)row_of<const T>(p.x, group(r), r - group(r) * p.rows) & 15) / (int)sizeof(T) : 0, p.dim};
  int count = 0;
  uint32_t edge = 0;  // vectors that the row has in part
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!units.live(t + i * L)) continue;
    ++count;
    if (SHIFT && !units.whole(t + i * L)) edge |= 1u << i;
  }
  const uint32_t whole = ((1u << count) - 1u) & ~edge;
  auto edges = [&](auto f) {
    if constexpr (SHIFT) {
      if (!edge) return;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (edge >> i & 1) f(i, t + i * L);
    }
  };
  pdl_wait();
  Raw<T, E> x[NV], res[NV];
  auto bring = [&](int64_t at) {
    const bool live = at < p.total;
    const int64_t g = group(at), gr = at - g * p.rows;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i].zero(), res[i].zero();
      if (live && i < count) {
        x[i].load(row_of<const T>(p.x, g, gr) + units.col(t + i * L));
        if (has_res) res[i].load(row_of<const T>(p.residual, g, gr) + units.col(t + i * L));
      }
    }
  };
  uint64_t w[HELD ? NV * P : P], b[HELD ? NV * P : P];
  int64_t held_of = -1;  // the group whose parameters w and b are
  auto params = [&](int64_t g, int i, int at) {
    const int c = t + i * L;
#pragma unroll
    for (int j = 0; j < P; ++j) b[at + j] = 0;
    if constexpr (SHIFT) {
      units.params(p.weight.data + g * p.weight.group, c, w + at);
      if (p.bias.data) units.params(p.bias.data + g * p.bias.group, c, b + at);
    } else {
      load_pairs<E>(p.weight.data + g * p.weight.group + c * E, w + at);
      if (p.bias.data) load_pairs<E>(p.bias.data + g * p.bias.group + c * E, b + at);
    }
  };
  bring(r);
  for (; r - sub < p.total; r += step) {  // (the same turns for all lanes of a warp)
    uint64_t v[NV * P];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      pairs_of<T, E>(x[i], v + i * P);
      if (has_res) {
        uint64_t u[P];
        pairs_of<T, E>(res[i], u);
#pragma unroll
        for (int j = 0; j < P; ++j) v[i * P + j] = add2(v[i * P + j], u[j]);
      }
    }
    edges([&](int i, int c) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float2 f = unpack2(v[i * P + j]);
        v[i * P + j] = pack2(units.in(c, 2 * j) ? f.x : 0.f, units.in(c, 2 * j + 1) ? f.y : 0.f);
      }
    });
    bring(r + step);
    const bool live = r < p.total;
    const int64_t g = group(r), gr = r - g * p.rows;
    if (p.sum.data || (!SHIFT && p.kept.data)) {
      T* s = p.sum.data ? row_of<T>(p.sum, g, gr) : nullptr;
      int8_t* q = p.kept.data + g * p.kept.group + gr * p.kept.row;
      uint8_t* scale = p.kept.scale + g * p.kept.scale_group + gr * p.kept.scale_row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Raw<T, E> u = rounded<T, E>(v + i * P);
        if (s && live && whole >> i & 1) store_raw<T, E>(s + units.col(t + i * L), u);
        if (!SHIFT && p.kept.data) keep_raw<T, E>(q, scale, (t + i * L) * E, live && i < count, u);
      }
      if (s && live) edges([&](int i, int c) { store_edge<T, E>(s, units, c, rounded<T, E>(v + i * P)); });
    }
    float sum = pairs_sum(v);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float mean = sum * p.inv_dim;
    float m2 = pairs_squares<E, NV>(v, mean, whole);
    edges([&](int i, int c) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 f = unpack2(v[i * P + e / 2]);
        const float off = (e & 1 ? f.y : f.x) - mean;
        if (units.in(c, e)) m2 = fmaf(off, off, m2);
      }
    });
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
    const Moments mo{mean, rsqrtf(fmaf(m2, p.inv_dim, p.eps))};
    if (HELD && g != held_of) {
      held_of = g;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) params(g, i, HELD ? i * P : 0);
    }
    if (t == 0 && live) {
      if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
      if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
    }
    if (p.scale.data) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) {
          if (!HELD) params(g, i, 0);
          const float here = pairs_affine<E, true>(v + i * P, mo, w + (HELD ? i * P : 0), b + (HELD ? i * P : 0), top);
          if (whole >> i & 1) top = here;
        }
      edges([&](int i, int c) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 f = unpack2(v[i * P + e / 2]);
          if (units.in(c, e)) top = max_nan(top, fabsf(e & 1 ? f.y : f.x));
        }
      });
      uint32_t most = __float_as_uint(top);
#pragma unroll
      for (int o = L / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
      const float scale = scale_of(__uint_as_float(most));
      const Reciprocal inv = reciprocal_of(scale);
      if (!live) continue;
      if (t == 0) p.scale.data[g * p.scale.group + gr] = scale;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (whole >> i & 1) store_pairs_e4m3<E>(row_of<e4m3>(p.y, g, gr) + units.col(t + i * L), v + i * P, inv);
      edges([&](int i, int c) { store_edge_e4m3<E>(row_of<e4m3>(p.y, g, gr), units, c, v + i * P, inv); });
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (live && i < count) {
          if (!HELD) params(g, i, 0);
          pairs_affine<E, false>(v + i * P, mo, w + (HELD ? i * P : 0), b + (HELD ? i * P : 0), 0.f);
          if (whole >> i & 1) store_pairs<T, E>(row_of<T>(p.y, g, gr) + units.col(t + i * L), v + i * P);
        }
      if (live) edges([&](int i, int c) { store_edge<T, E>(row_of<T>(p.y, g, gr), units, c, rounded<T, E>(v + i * P)); });
    }
  }
}

// ---- many rows: a block of one row's threads walks over rows that arrive in a ring of shared-memory stages by bulk
// copies, so that loads stay in flight while rows are summed and written.
//
// SHIFT: rows off the 16-byte grid (odd widths), all of a call's matrices at the same place of a unit in each row. A
// thread takes whole units, the row's first and last in part. A block's rows lie a multiple of 16 rows' bytes apart, so
// that all of them begin at the same place of a unit: weights and biases stand in shared memory in those units. (For
// rows at any place, a word to each column, bf16 16385 x 4097 took 128 us; in registers, which leave room for fewer
// blocks, 194; so 97.)
template <typename T, int E, int NV, bool SHIFT>
__global__ void __launch_bounds__(512, E * NV == 16 || E == 8 ? 2 : 1)
    k_layer_stream(const LayerArgs p, int stages, int slot, int* err) {
  constexpr int P = E / 2;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float4 s_share[2][16];
  __shared__ uint32_t s_top[2][16];
  const bool has_res = p.residual.data;
  const Ring q = ring_init(smem, stages, slot, has_res ? 2 : 1);
  const int t = threadIdx.x, tpr = blockDim.x, bytes = p.dim * (int)sizeof(T);
  const int warp = t >> 5, warps = tpr >> 5;
  const int64_t rows = SHIFT ? p.rows : p.total, g0 = SHIFT ? blockIdx.y : 0;  // (SHIFT: of one group)
  auto place = [&](int64_t r, int64_t& g, int64_t& gr) {
    g = SHIFT ? g0 : group_at(r, p.rows, p.total);
    gr = SHIFT ? r : r - g * p.rows;
  };
  const Units<E> units{SHIFT ? (int)((uint64_t)row_of<const T>(p.x, g0, blockIdx.x) & 15) / (int)sizeof(T) : 0, p.dim};
  int count = 0, held = 0;
  uint32_t edge = 0;  // vectors that the row has in part
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * tpr;
    if (!units.live(c)) continue;
    ++count;
    held += SHIFT ? units.count(c) : E;
    if (SHIFT && !units.whole(c)) edge |= 1u << i;
  }
  const uint32_t whole = ((1u << count) - 1u) & ~edge;
  // (few threads have any: apart from the others' code, whose instructions bound bf16 rows)
  auto edges = [&](auto f) {
    if constexpr (SHIFT) {
      if (!edge) return;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (edge >> i & 1) f(i);
    }
  };
  const float n = (float)__reduce_add_sync(0xffffffffu, held), inv_n = n > 0.f ? 1.f / n : 0.f;
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    int64_t g, gr;
    place(r, g, gr);
    const char* src[3] = {(const char*)row_of<const T>(p.x, g, gr),
                          has_res ? (const char*)row_of<const T>(p.residual, g, gr) : nullptr, nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < rows) load(r, s);
    }
  // [quarters of a unit][weights, biases][units of the row][4], zeros beside the row (so that lanes read adjacent 16 bytes)
  float* s_par = reinterpret_cast<float*>(smem + RING_BARS + stages * q.arrays * slot);
  const int width = (int)(units.m + p.dim + E - 1) / E * E, plane = width / E * 4;
  if constexpr (SHIFT) {
    const float* w = p.weight.data + g0 * p.weight.group;
    const float* b = p.bias.data ? p.bias.data + g0 * p.bias.group : nullptr;
    for (int i = t; i < width; i += tpr) {
      const int c = i - units.m;
      const bool in = c >= 0 && c < p.dim;
      float* to = s_par + i % E / 4 * 2 * plane + i / E * 4 + i % 4;
      to[0] = in ? __ldg(w + c) : 0.f, to[plane] = in && b ? __ldg(b + c) : 0.f;
    }
    __syncthreads();
  }
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    int64_t g, gr;
    place(r, g, gr);
    const char* at = reinterpret_cast<const char*>(smem) + RING_BARS + stage * q.arrays * slot;
    const T* x = reinterpret_cast<const T*>(at + (SHIFT ? 0 : (uint64_t)row_of<const T>(p.x, g, gr) & 15));
    const T* res = reinterpret_cast<const T*>(
        at + slot + (SHIFT ? 0 : has_res ? (uint64_t)row_of<const T>(p.residual, g, gr) & 15 : 0));
    ring_wait(q, stage, turn & 1);
    uint64_t v[NV * P];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (i < count) {
        Raw<T, E> a;
        a.load(x + (t + i * tpr) * E);
        pairs_of<T, E>(a, v + i * P);
        if (has_res) {
          uint64_t u[P];
          a.load(res + (t + i * tpr) * E);
          pairs_of<T, E>(a, u);
#pragma unroll
          for (int j = 0; j < P; ++j) v[i * P + j] = add2(v[i * P + j], u[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < P; ++j) v[i * P + j] = 0;
      }
    }
    edges([&](int i) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float2 f = unpack2(v[i * P + j]);
        v[i * P + j] = pack2(units.in(t + i * tpr, 2 * j) ? f.x : 0.f, units.in(t + i * tpr, 2 * j + 1) ? f.y : 0.f);
      }
    });
    const float sum = warp_sum(pairs_sum(v)), own = sum * inv_n;
    float m2 = pairs_squares<E, NV>(v, own, whole);
    edges([&](int i) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 f = unpack2(v[i * P + e / 2]);
        const float off = (e & 1 ? f.y : f.x) - own;
        if (units.in(t + i * tpr, e)) m2 = fmaf(off, off, m2);
      }
    });
    m2 = warp_sum(m2);
    float4* shares = s_share[turn >> 1 & 1];
    if ((t & 31) == 0) shares[warp] = make_float4(n, sum, own, m2);
    __syncthreads();
    // (the row is in registers everywhere: its stage takes the row that comes `stages` later)
    if (t == 0 && r + (int64_t)stages * gridDim.x < rows) load(r + (int64_t)stages * gridDim.x, stage);
    if (p.sum.data || (!SHIFT && p.kept.data)) {
      T* s = p.sum.data ? row_of<T>(p.sum, g, gr) : nullptr;
      int8_t* kq = p.kept.data + g * p.kept.group + gr * p.kept.row;
      uint8_t* scale = p.kept.scale + g * p.kept.scale_group + gr * p.kept.scale_row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Raw<T, E> u = rounded<T, E>(v + i * P);
        const int c = t + i * tpr;
        if (s && whole >> i & 1) store_raw<T, E>(s + units.col(c), u);
        if (!SHIFT && p.kept.data) keep_raw<T, E>(kq, scale, c * E, i < count, u);
      }
      edges([&](int i) { store_edge<T, E>(s, units, t + i * tpr, rounded<T, E>(v + i * P)); });
    }
    const Moments mo = join_shares(shares, warps, p.inv_dim, p.eps);
    if (t == 0) {
      if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
      if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
    }
    const float* weight = p.weight.data + g * p.weight.group;
    const float* bias = p.bias.data ? p.bias.data + g * p.bias.group : nullptr;
    auto params = [&](int i, uint64_t* w, uint64_t* b) {
      if constexpr (SHIFT) {
#pragma unroll
        for (int j = 0; j < P; j += 2) {
          const float* from = s_par + j / 2 * 2 * plane + (t + i * tpr) * 4;
          const ulonglong2 x2 = *reinterpret_cast<const ulonglong2*>(from);
          const ulonglong2 y2 = *reinterpret_cast<const ulonglong2*>(from + plane);
          w[j] = x2.x, w[j + 1] = x2.y, b[j] = y2.x, b[j + 1] = y2.y;
        }
      } else {
        load_pairs<E>(weight + (t + i * tpr) * E, w);
#pragma unroll
        for (int j = 0; j < P; ++j) b[j] = 0;
        if (bias) load_pairs<E>(bias + (t + i * tpr) * E, b);
      }
    };
    if (p.scale.data) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) {
          uint64_t w[P], b[P];
          params(i, w, b);
          const float here = pairs_affine<E, true>(v + i * P, mo, w, b, top);
          if (whole >> i & 1) top = here;
        }
      edges([&](int i) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 f = unpack2(v[i * P + e / 2]);
          if (units.in(t + i * tpr, e)) top = max_nan(top, fabsf(e & 1 ? f.y : f.x));
        }
      });
      uint32_t* tops = s_top[turn >> 1 & 1];
      uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
      if ((t & 31) == 0) tops[warp] = most;
      __syncthreads();
      most = __reduce_max_sync(0xffffffffu, tops[min(t & 31, warps - 1)]);
      const float scale = scale_of(__uint_as_float(most));
      const Reciprocal inv = reciprocal_of(scale);
      if (t == 0) p.scale.data[g * p.scale.group + gr] = scale;
      e4m3* y = row_of<e4m3>(p.y, g, gr);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (whole >> i & 1) store_pairs_e4m3<E>(y + units.col(t + i * tpr), v + i * P, inv);
      edges([&](int i) { store_edge_e4m3<E>(y, units, t + i * tpr, v + i * P, inv); });
    } else {
      T* y = row_of<T>(p.y, g, gr);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) {
          uint64_t w[P], b[P];
          params(i, w, b);
          pairs_affine<E, false>(v + i * P, mo, w, b, 0.f);
          if (whole >> i & 1) store_pairs<T, E>(y + units.col(t + i * tpr), v + i * P);
        }
      edges([&](int i) { store_edge<T, E>(y, units, t + i * tpr, rounded<T, E>(v + i * P)); });
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
}

// One wave of blocks, whose turns are a multiple of 8 rows.
template <typename T, int E, int NV, int L, bool SHIFT>
cudaError_t launch_short(const LayerArgs& p, cudaStream_t st) {
  constexpr auto kernel = k_layer_short<T, E, NV, L, SHIFT>;
  static const int resident = [] {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, 32 * SHORT_WARPS, 0);
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess && n > 0 ? n : 4;
  }();
  const int64_t most = (int64_t)sm_count() * resident, want = ceil_div(p.total, SHORT_WARPS * (32 / L));
  const int64_t blocks = want < most ? want : (most + 1) / 2 * 2;
  return launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * SHORT_WARPS), 0, st, p);
}
template <typename T, int E, bool SHIFT>
cudaError_t launch_short(const LayerArgs& p, int lanes, cudaStream_t st) {
  if (lanes <= 4) return launch_short<T, E, 16 / E, 4, SHIFT>(p, st);
  if (lanes <= 8) return launch_short<T, E, 16 / E, 8, SHIFT>(p, st);
  if (lanes <= 16) return launch_short<T, E, 16 / E, 16, SHIFT>(p, st);
  return launch_short<T, E, 16 / E, 32, SHIFT>(p, st);
}

// Blocks of a group (shift: whose rows must begin at the same place of a unit, 16 bytes' rows apart or alone).
int64_t shift_blocks(int64_t blocks, int64_t rows, int u) {
  if (blocks >= rows) return rows;
  return blocks < u ? (rows < u ? rows : u) : blocks - blocks % u;
}

template <auto KERNEL>
cudaError_t launch_rings(const LayerArgs& p, StreamShape s, int shift, cudaStream_t st) {
  const cudaError_t e = allow_smem<KERNEL>();
  if (e != cudaSuccess) return e;
  static const int registers = registers_of((const void*)KERNEL);
  s.per_sm = blocks_resident(registers, s.tpr, s.per_sm);
  s.fit();
  const int64_t groups = p.total / p.rows, fill = (int64_t)s.per_sm * sm_count();
  const dim3 grid = shift ? dim3((unsigned)shift_blocks(ceil_div(fill, groups), p.rows, shift), (unsigned)groups)
                          : dim3((unsigned)(fill < p.total ? fill : p.total));
  return launch_pdl(KERNEL, grid, dim3(s.tpr), s.smem, st, p, s.stages, s.slot, timeout_word());
}

// Whether rows go by units: off the 16-byte grid, at the same place of a unit in all of the matrices.
bool layer_shift(const LayerArgs& p) {
  const int e = 16 / type_bytes(p.x.type);
  const int64_t groups = p.total / p.rows;
  return p.total > STREAM_ROWS * sm_count() && p.dim <= SHIFT_DIM && same_shift(p.x, p.y, groups, p.rows, e) &&
         same_shift(p.x, p.residual, groups, p.rows, e) && same_shift(p.x, p.sum, groups, p.rows, e);
}

template <typename T, int E>
cudaError_t launch_layer(LayerArgs& p, cudaStream_t st) {
  constexpr int U = 16 / sizeof(T);
  const bool many = p.total > STREAM_ROWS * sm_count();
  const int arrays = p.residual.data ? 2 : 1;
  if constexpr (E > 1) {
    const int lanes = (int)ceil_div(p.dim, 16);
    if (many && lanes <= 32) return launch_short<T, E, false>(p, lanes, st);
    if (many && lanes <= 64) return launch_short<T, E, 32 / E, 32, false>(p, st);
    if (many) {
      // bf16 rows in 32 elements per thread where one matrix alone keeps the loads going, and to 8 bits, whose second
      // barrier costs a block of many warps more: 16384 x 4096 without residual 60 us (of 16 elements 71), with it 114
      // (101, kept in 8 bits), 16384 x 8192 to 8 bits 188 (208), kept in 8 bits 221 (204).
      const bool wide = E == 8 && (!p.residual.data || (p.scale.data && p.dim > 4096));
      const StreamShape s = stream_shape(p.dim, E, sizeof(T), arrays, 2048, 0, wide);
      return s.wide ? launch_rings<k_layer_stream<T, E, 32 / E, false>>(p, s, 0, st)
                    : launch_rings<k_layer_stream<T, E, 16 / E, false>>(p, s, 0, st);
    }
  } else if (layer_shift(p)) {
    // (a row touches a unit more than it fills)
    // (rows of several groups are one sequence to k_layer_short, which must begin as one group's do)
    const int lanes = (int)ceil_div(p.dim + U - 1, 16);
    if (lanes <= 32 && (p.total == p.rows || (p.x.group - p.rows * p.x.row) % U == 0))
      return launch_short<T, U, true>(p, lanes, st);
    // (of 32 elements per thread bf16 rows have no registers left: 16385 x 4097 172 us)
    const int wide = (int)ceil_div(p.dim + U - 1, U) * U;
    StreamShape s = stream_shape(wide, U, sizeof(T), arrays, 2048);
    s.fixed = 2 * wide * 4;
    s.share(2048);
    return launch_rings<k_layer_stream<T, U, 16 / U, true>>(p, s, U, st);
  }
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

// Where a block's sums go: its part, or the results themselves.
struct SumsOut {
  float *dw, *db;
};
__device__ __forceinline__ SumsOut sums_out(const LayerBack& p, int64_t g) {
  if (p.part) {
    float* dw = p.part + (g * gridDim.x + blockIdx.x) * 2 * p.dim;
    return {dw, dw + p.dim};
  }
  return {p.dweight.data ? p.dweight.data + g * p.dweight.group : nullptr,
          p.dbias.data ? p.dbias.data + g * p.dbias.group : nullptr};
}

// Rows whose matrices lie at different places of a 16-byte unit, element by element: a block of one row's threads
// walks over rows of one group (blockIdx.y); the sums over its rows stay in registers.
template <typename T, int NV, bool KEPT>
__global__ void __launch_bounds__(512) k_layer_backward(const LayerBack p) {
  __shared__ float2 s_red[2][16];
  constexpr int E = 1;
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
        s[i][0] = (float)*q * unit;
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
  const SumsOut out = sums_out(p, g);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (t + i * tpr < nvec) {
      if (out.dw) out.dw[t + i * tpr] = dw[i][0];
      if (out.db) out.db[t + i * tpr] = db[i][0];
    }
}

// Two sums over a warp: afterwards a on lanes 0 to 15, b on the others.
__device__ __forceinline__ float warp_pair(float a, float b) {
  const bool high = threadIdx.x & 16;
  float v = (high ? b : a) + __shfl_xor_sync(0xffffffffu, high ? a : b, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// N pairs of sums as a tree, all loads in flight at once (one after the other 16384 x 8192 with dsum 190 us, so 184).
template <int N>
__device__ __forceinline__ uint64_t sum_places(const float2* s) {
  uint64_t v[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const ulonglong2 q = reinterpret_cast<const ulonglong2*>(s)[i];
    v[i] = add2(q.x, q.y);
  }
#pragma unroll
  for (int o = N / 4; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) v[i] = add2(v[i], v[i + o]);
  return v[0];
}
// A team's two sums, with one barrier (its own, `id`); s: a place per warp, by turns.
__device__ __forceinline__ float2 team_sum(float2 v, float2* s, int warp, int warps, int id) {
  const float w = warp_pair(v.x, v.y);
  if (warps == 1) return make_float2(__shfl_sync(0xffffffffu, w, 0), __shfl_sync(0xffffffffu, w, 16));
  if ((threadIdx.x & 15) == 0) (&s[warp].x)[threadIdx.x >> 4 & 1] = w;
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
  if (warps == 8) return unpack2(sum_places<8>(s));
  if (warps == 16) return unpack2(sum_places<16>(s));
  const uint64_t* pairs = reinterpret_cast<const uint64_t*>(s);
  uint64_t r = pairs[0];
#pragma unroll 4
  for (int i = 1; i < warps; ++i) r = add2(r, pairs[i]);
  return unpack2(r);
}

// A vector of what was normalised, as it lies in memory: of dy's type, or a checkpoint's multiples and their unit (SHIFT:
// from a column that need not be a block's, so that the last `behind` elements may have another).
template <typename T, int E, bool KEPT, bool SHIFT = false>
struct Source {
  Raw<T, E> raw;
  __device__ __forceinline__ void zero() { raw.zero(); }
  __device__ __forceinline__ void clear(int e) { raw.clear(e); }
  __device__ __forceinline__ void get(uint64_t* v) const { pairs_of<T, E>(raw, v); }
};
template <typename T, int E, bool SHIFT>
struct Source<T, E, true, SHIFT> {
  static_assert(E >= 4, "words");
  uint32_t w[E / 4];  // multiples + 128
  float unit, unit2;
  int border;  // SHIFT: elements before it have the first unit
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : w) v = 0;
    unit = unit2 = 0.f;
    border = E;
  }
  __device__ __forceinline__ void clear(int e) { w[e / 4] = (w[e / 4] & ~(255u << e % 4 * 8)) | 128u << e % 4 * 8; }
  __device__ __forceinline__ void load(const int8_t* q, uint32_t byte) {
    if constexpr (E == 8) {
      const uint2 r = *reinterpret_cast<const uint2*>(q);
      w[0] = r.x ^ 0x80808080u, w[1] = r.y ^ 0x80808080u;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(q) ^ 0x80808080u;
    }
    unit = block_unit(byte);
  }
  // From shared memory, at any byte, up to E - 1 of them before the row.
  __device__ __forceinline__ void load(const uint8_t* q, const uint8_t* scale, int col, int dim) {
    const uint8_t* from = q + col;
    const uint32_t off = (uint32_t)(uint64_t)from & 3u;
    const uint32_t* words = reinterpret_cast<const uint32_t*>(from - off);
    uint32_t r[E / 4 + 1];
#pragma unroll
    for (int j = 0; j <= E / 4; ++j) r[j] = words[j];
#pragma unroll
    for (int j = 0; j < E / 4; ++j) w[j] = __funnelshift_r(r[j], r[j + 1], off * 8) ^ 0x80808080u;
    const int first = max(col, 0), last = min(col + E, dim) - 1;
    unit = block_unit(scale[first / LIPZ_BLOCK]), unit2 = block_unit(scale[last / LIPZ_BLOCK]);
    border = (first | (LIPZ_BLOCK - 1)) + 1 - col;
  }
  // From global memory, at any byte.
  __device__ __forceinline__ void gather(const int8_t* q, const uint8_t* scale, int col, int dim) {
    if (col >= 0 && col + E <= dim) {
      const uint4 r = bytes16(reinterpret_cast<const uint8_t*>(q) + col, E);
      const uint32_t two[2] = {r.x, r.y};
#pragma unroll
      for (int j = 0; j < E / 4; ++j) w[j] = two[j] ^ 0x80808080u;
    } else {
#pragma unroll
      for (int j = 0; j < E / 4; ++j) w[j] = 0x80808080u;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (col + e >= 0 && col + e < dim) w[e / 4] ^= (uint32_t)(uint8_t)__ldg(q + col + e) << e % 4 * 8;
    }
    const int first = max(col, 0), last = min(col + E, dim) - 1;
    unit = block_unit(__ldg(scale + first / LIPZ_BLOCK)), unit2 = block_unit(__ldg(scale + last / LIPZ_BLOCK));
    border = (first | (LIPZ_BLOCK - 1)) + 1 - col;
  }
  __device__ __forceinline__ void get(uint64_t* v) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const uint64_t a = pack2(__uint_as_float(__byte_perm(w[i / 2], 0x4B000000u, i & 1 ? 0x7442 : 0x7440)),
                               __uint_as_float(__byte_perm(w[i / 2], 0x4B000000u, i & 1 ? 0x7443 : 0x7441)));
      const uint64_t by = SHIFT ? pack2(2 * i < border ? unit : unit2, 2 * i + 1 < border ? unit : unit2) : both(unit);
      v[i] = mul2(add2(a, both(-8388736.f)), by);
    }
  }
};

// A vector's terms (x: s - mean): of the two sums along the row (g, and g x) and of those down the columns.
struct Terms {
  uint64_t along_g = 0, along_x = 0;
  __device__ __forceinline__ float2 sums() const {
    const float2 a = unpack2(along_g), b = unpack2(along_x);
    return make_float2(a.x + a.y, b.x + b.y);
  }
};
template <int E>
__device__ __forceinline__ void take_mean(uint64_t* s, float mean) {
#pragma unroll
  for (int j = 0; j < E / 2; ++j) s[j] = add2(s[j], both(-mean));
}
template <typename T, int E>
__device__ __forceinline__ void add_terms(Terms& t, const Raw<T, E>& dy, const uint64_t* x, const uint64_t* w,
                                          float rstd, uint64_t* dw, uint64_t* db) {
  uint64_t d[E / 2];
  pairs_of<T, E>(dy, d);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const uint64_t m = mul2(d[j], x[j]);
    dw[j] = fma2(m, both(rstd), dw[j]);
    db[j] = add2(d[j], db[j]);
    t.along_g = fma2(d[j], w[j], t.along_g);
    t.along_x = fma2(m, w[j], t.along_x);
  }
}
// dx = rstd (g - c1 - (s - mean) c2) + dsum
template <typename T, int E>
__device__ __forceinline__ void gradient(uint64_t* v, const Raw<T, E>& dy, const uint64_t* x, const uint64_t* w,
                                         const Raw<T, E>& ds, float rstd, float c1, float c2) {
  uint64_t d[E / 2];
  pairs_of<T, E>(dy, d);
  pairs_of<T, E>(ds, v);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const uint64_t a = fma2(x[j], both(-c2), fma2(d[j], w[j], both(-c1)));
    v[j] = fma2(both(rstd), a, v[j]);
  }
}

// Where a stage's rows stand, and how many bytes one has: of dy, of what was normalised, of its scales, of dsum.
struct BackStage {
  int at[4], bytes[4];
};
__device__ __forceinline__ void load_stage(const Ring& q, const BackStage& b, int stage, const void* const* src) {
  uint32_t total = 0;
  uint64_t from[4];
  uint32_t size[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t a = (uint64_t)src[i];
    from[i] = a & ~15ull;
    size[i] = b.bytes[i] ? (uint32_t)(((a + b.bytes[i] + 15) & ~15ull) - from[i]) : 0u;
    total += size[i];
  }
  const uint32_t bar = q.bars + 8 * stage;
  tc::mbar_expect_tx(bar, total);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (size[i])
      asm volatile(
          "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
              q.data + stage * q.slot + b.at[i]),
          "l"(from[i]), "r"(size[i]), "r"(bar)
          : "memory");
}
// The rows' addresses in memory.
template <typename T, bool KEPT>
__device__ __forceinline__ void back_rows(const LayerBack& p, int64_t g, int64_t r, const void** src) {
  src[0] = row_of<const T>(p.dy, g, r);
  if constexpr (KEPT) {
    src[1] = p.kept.data + g * p.kept.group + r * p.kept.row;
    src[2] = p.kept.scale + g * p.kept.scale_group + r * p.kept.scale_row;
  } else {
    src[1] = row_of<const T>(p.s, g, r);
    src[2] = nullptr;
  }
  src[3] = p.dsum.data ? row_of<const T>(p.dsum, g, r) : nullptr;
}

// Teams of one row's threads, several to a block, walk over rows of one group (blockIdx.y), which arrive in a ring of
// each; their sums for dweight and dbias stay in registers, and of 16 elements the weights. At the end the teams' sums
// are added in shared memory: one part per SM is left for the launch that adds those (16384 x 2048 over a checkpoint:
// with a part per team 65 us, 7 of them that launch; so 62). SHIFT: rows off the 16-byte grid, as in k_layer_stream; a
// checkpoint's row lies at any byte: its multiples come from the words that hold them, and a unit's columns from two
// blocks at most.
//
// Bound: latency at 16 warps of 128 registers. 8192 x 4096 with dsum takes 51 us by itself, with DRAM in use for 61 % of
// them and half of the issue slots: between two instructions a warp waits for the one before (1.7 clocks), at the row's
// barrier (1.5) and for shared memory (1.5). An element takes 26 instructions, of which about nine are its arithmetic and
// conversions (two elements at a time where the instruction exists); the rest is a row's: reduction, barrier, ring, moves.
// Two rows of a team at once took 74, rows read again in the place of registers 62 (640 threads), 8 elements per thread 79.
constexpr int TEAM_THREADS = 512;  // of a block (registers)

template <typename T, int E, int NV, bool KEPT, bool SHIFT>
__global__ void __launch_bounds__(TEAM_THREADS) k_layer_back_stream(const LayerBack p, const BackStage b, int tpr, int stages,
                                                           int slot, int* err) {
  constexpr int P = E / 2;
  constexpr bool HELD = NV * E == 16;
  static_assert(!SHIFT || HELD, "weights in registers");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(16) float2 s_red[2][TEAM_THREADS / 32];
  const bool has_dsum = p.dsum.data;
  const int teams = blockDim.x / tpr, team = threadIdx.x / tpr, t = threadIdx.x - team * tpr, warps = tpr >> 5;
  const int ring_bytes = RING_BARS + stages * slot;
  uint8_t* ring = smem + team * ring_bytes;
  const Ring q = ring_of(ring, stages, slot, 1);
  if (t == 0) ring_set_up(q);
  __syncthreads();
  const int64_t g = blockIdx.y, first = (int64_t)blockIdx.x * teams + team, step = (int64_t)gridDim.x * teams;
  const Units<E> units{SHIFT ? (int)((uint64_t)row_of<const T>(p.dy, g, first) & 15) / (int)sizeof(T) : 0, p.dim};
  int count = 0;
  bool edge = false;  // the row has some of this thread's vectors in part
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * tpr;
    if (!units.live(c)) continue;
    ++count;
    if (SHIFT && !units.whole(c)) edge = true;
  }
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const void* src[4];
    back_rows<T, KEPT>(p, g, r, src);
    load_stage(q, b, stage, src);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = first + s * step;
      if (r < p.rows) load(r, s);
    }
  const float* weight = p.weight.data + g * p.weight.group;
  uint64_t dw[NV][P], db[NV][P], hw[HELD ? NV : 1][P];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < P; ++j) dw[i][j] = db[i][j] = 0;
    if constexpr (HELD) {
      if (SHIFT) units.params(weight, t + i * tpr, hw[i]);
      else if (i < count) load_pairs<E>(weight + (t + i * tpr) * E, hw[i]);
    }
  }
  const float *means = p.mean.data + g * p.mean.group, *rstds = p.rstd.data + g * p.rstd.group;
  float next_mean = 0.f, next_rstd = 0.f;  // (of the row after this one: in flight while this one is worked on)
  if (first < p.rows) next_mean = __ldg(means + first), next_rstd = __ldg(rstds + first);
  // a checkpoint's rows begin anywhere in their 16-byte units
  uint32_t low_q = 0, low_scale = 0, step_q = 0, step_scale = 0;
  if constexpr (KEPT) {
    low_q = (uint32_t)(uint64_t)(p.kept.data + g * p.kept.group + first * p.kept.row);
    low_scale = (uint32_t)(uint64_t)(p.kept.scale + g * p.kept.scale_group + first * p.kept.scale_row);
    step_q = (uint32_t)(step * p.kept.row), step_scale = (uint32_t)(step * p.kept.scale_row);
  }
  T* dx = row_of<T>(p.dx, g, first);
  const int64_t dx_step = step * p.dx.row;
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = first; r < p.rows; r += step) {
    const float mean = next_mean, rstd = next_rstd;
    if (r + step < p.rows) next_mean = __ldg(means + r + step), next_rstd = __ldg(rstds + r + step);
    const uint8_t* at = ring + RING_BARS + stage * slot;
    const uint8_t *at_q = at + b.at[1] + (low_q & 15), *at_scale = at + b.at[2] + (low_scale & 15);
    ring_wait(q, stage, turn & 1);
    // A vector of dy and of what was normalised; zeros where neither is the row's (what lies beside it adds nothing).
    auto take = [&](int i, Raw<T, E>& dy, uint64_t* v) {
      const int c = t + i * tpr;
      Source<T, E, KEPT, SHIFT> x;
      dy.load(reinterpret_cast<const T*>(at + b.at[0]) + c * E);
      if constexpr (KEPT && SHIFT)
        x.load(at_q, at_scale, units.col(c), p.dim);
      else if constexpr (KEPT)
        x.load(reinterpret_cast<const int8_t*>(at_q) + c * E, at_scale[c * E / LIPZ_BLOCK]);
      else
        x.raw.load(reinterpret_cast<const T*>(at + b.at[1]) + c * E);
      if (SHIFT && edge) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!units.in(c, e)) dy.clear(e), x.clear(e);
      }
      x.get(v);
      take_mean<E>(v, mean);
    };
    Terms terms;
    Raw<T, E> dy[HELD ? NV : 1];
    uint64_t x[HELD ? NV : 1][P];
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        const int h = HELD ? i : 0;
        take(i, dy[h], x[h]);
        uint64_t w[P];
        if constexpr (!HELD) load_pairs<E>(weight + (t + i * tpr) * E, w);
        add_terms<T, E>(terms, dy[h], x[h], HELD ? hw[h] : w, rstd, dw[i], db[i]);
      }
    const float2 along = team_sum(terms.sums(), s_red[turn >> 1 & 1] + team * warps, t >> 5, warps, team + 1);
    // (every thread is done with the row before this one, whose stage takes the row that comes stages - 1 later: until
    // then dsum is read from there, and of 32 elements all, which registers do not hold over the barrier)
    if (t == 0 && stages > 1 && r != first && r + (stages - 1) * step < p.rows)
      load(r + (stages - 1) * step, stage ? stage - 1 : stages - 1);
    // (rstd^2 by itself may be infinite where the gradient is not)
    const float c1 = along.x * p.inv_dim, c2 = rstd * (rstd * (along.y * p.inv_dim));
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        const int c = t + i * tpr;
        const int h = HELD ? i : 0;
        Raw<T, E> ds;
        uint64_t w[P], v[P];
        ds.zero();
        if (has_dsum) ds.load(reinterpret_cast<const T*>(at + b.at[3]) + c * E);
        if constexpr (!HELD) {
          take(i, dy[0], x[0]);
          load_pairs<E>(weight + c * E, w);
        }
        gradient<T, E>(v, dy[h], x[h], HELD ? hw[h] : w, ds, rstd, c1, c2);
        if (SHIFT && edge && !units.whole(c)) store_edge<T, E>(dx, units, c, rounded<T, E>(v));
        else store_pairs<T, E>(dx + units.col(c), v);
      }
    if (stages == 1) {  // (rows of which shared memory holds one)
      asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(tpr) : "memory");
      if (t == 0 && r + step < p.rows) load(r + step, 0);
    }
    dx += dx_step;
    low_q += step_q, low_scale += step_scale;
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  __syncthreads();
  int code = 0;  // a wait that expired: copies in flight land before the block leaves, or its rings are written over
  for (int k = 0; k < teams; ++k)
    if (*reinterpret_cast<volatile int*>(smem + k * ring_bytes + 8 * RING_MAX))
      code = *reinterpret_cast<volatile int*>(smem + k * ring_bytes + 8 * RING_MAX + 4);
  if (code) {
    const unsigned long long t0 = tc::globaltimer();
    while (tc::globaltimer() - t0 < 200000ull) {
    }
    if (threadIdx.x == 0 && err) *reinterpret_cast<volatile int*>(err) = code;
  }
  if (!p.dweight.data && !p.dbias.data) return;
  const SumsOut out = sums_out(p, g);
  float* s_sums = reinterpret_cast<float*>(smem);  // [teams][2][dim], over the rings
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < count)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = units.col(t + i * tpr) + e;
        const float2 a = unpack2(dw[i][e / 2]), d = unpack2(db[i][e / 2]);
        if (SHIFT && !units.in(t + i * tpr, e)) continue;
        if (teams > 1) {
          s_sums[team * 2 * p.dim + c] = e & 1 ? a.y : a.x, s_sums[(team * 2 + 1) * p.dim + c] = e & 1 ? d.y : d.x;
          continue;
        }
        if (out.dw) out.dw[c] = e & 1 ? a.y : a.x;
        if (out.db) out.db[c] = e & 1 ? d.y : d.x;
      }
  if (teams == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * p.dim; c += blockDim.x) {
    float v = 0.f;
#pragma unroll 4
    for (int k = 0; k < teams; ++k) v += s_sums[k * 2 * p.dim + c];
    if (c < p.dim && out.dw) out.dw[c] = v;
    if (c >= p.dim && out.db) out.db[c - p.dim] = v;
  }
}

// Short rows: L lanes to a row, 32 / L rows to a warp, loaded into registers one set ahead; a block of WARPS walks over
// rows of one group, and its warps' sums are added in shared memory; where a block takes a whole group these are the
// results, without a second launch (144 groups of 100 x 256, 30 MB: 6.2 us in a graph).
constexpr int BACK_WARPS = 16;  // (registers)

// SHIFT: rows off the 16-byte grid, as in k_layer_short: the columns of a warp's rows are different lanes', so that the
// sums of each of them meet in shared memory.
template <typename T, int E, int NV, int L, bool KEPT, bool SHIFT>
__global__ void __launch_bounds__(32 * BACK_WARPS) k_layer_back_short(const LayerBack p) {
  constexpr int WARPS = BACK_WARPS, R = 32 / L;
  constexpr int SETS = SHIFT ? WARPS * R : WARPS;
  extern __shared__ float s_sums[];  // [SETS][2][dim]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane % L, sub = lane / L;
  const int64_t g = blockIdx.y, step = (int64_t)gridDim.x * WARPS * R;
  int64_t r = ((int64_t)blockIdx.x * WARPS + warp) * R + sub;
  const Units<E> units{SHIFT ? (int)((uint64_t)row_of<const T>(p.dy, g, r) & 15) / (int)sizeof(T) : 0, p.dim};
  int count = 0;
  bool edge = false;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!units.live(t + i * L)) continue;
    ++count;
    if (SHIFT && !units.whole(t + i * L)) edge = true;
  }
  pdl_wait();
  constexpr int P = E / 2;
  uint64_t w[NV][P], dw[NV][P], db[NV][P];
  const float* weight = p.weight.data + g * p.weight.group;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < P; ++j) w[i][j] = dw[i][j] = db[i][j] = 0;
    if (SHIFT) units.params(weight, t + i * L, w[i]);
    else if (i < count) load_pairs<E>(weight + (t + i * L) * E, w[i]);
  }
  const bool has_dsum = p.dsum.data;
  Raw<T, E> dy[NV], ds[NV];
  Source<T, E, KEPT, SHIFT> x[NV];
  float mean = 0.f, rstd = 0.f;
  auto load = [&](int64_t r) {
    if (r >= p.rows) {  // (a row of zeros adds nothing to the sums)
      mean = rstd = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) dy[i].zero(), x[i].zero();
      return;
    }
    mean = p.mean.data[g * p.mean.group + r], rstd = p.rstd.data[g * p.rstd.group + r];
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        const int c = units.col(t + i * L);
        dy[i].load(row_of<const T>(p.dy, g, r) + c);
        if constexpr (KEPT && SHIFT)
          x[i].gather(p.kept.data + g * p.kept.group + r * p.kept.row,
                      p.kept.scale + g * p.kept.scale_group + r * p.kept.scale_row, c, p.dim);
        else if constexpr (KEPT)
          x[i].load(p.kept.data + g * p.kept.group + r * p.kept.row + c,
                    p.kept.scale[g * p.kept.scale_group + r * p.kept.scale_row + c / LIPZ_BLOCK]);
        else
          x[i].raw.load(row_of<const T>(p.s, g, r) + c);
        if (has_dsum) ds[i].load(row_of<const T>(p.dsum, g, r) + c);
        if (SHIFT && edge) {  // (what lies beside the row adds nothing, whatever it is)
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (!units.in(t + i * L, e)) dy[i].clear(e), x[i].clear(e);
        }
      }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) dy[i].zero(), x[i].zero(), ds[i].zero();
  load(r);
  for (; r - sub < p.rows; r += step) {  // (the same turns for all lanes of a warp)
    Raw<T, E> a[NV], c3[NV];
    Source<T, E, KEPT, SHIFT> y[NV];
    const float m = mean, f = rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i) a[i] = dy[i], y[i] = x[i], c3[i] = ds[i];
    load(r + step);
    Terms terms;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        uint64_t s[P];
        y[i].get(s);
        take_mean<E>(s, m);
        add_terms<T, E>(terms, a[i], s, w[i], f, dw[i], db[i]);
      }
    float2 along = terms.sums();
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
      along.x += __shfl_xor_sync(0xffffffffu, along.x, o);
      along.y += __shfl_xor_sync(0xffffffffu, along.y, o);
    }
    if (r >= p.rows) continue;
    const float c1 = along.x * p.inv_dim, c2 = f * (f * (along.y * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        uint64_t s[P], v[P];
        y[i].get(s);
        take_mean<E>(s, m);
        gradient<T, E>(v, a[i], s, w[i], c3[i], f, c1, c2);
        if (SHIFT && edge && !units.whole(t + i * L)) store_edge<T, E>(dx, units, t + i * L, rounded<T, E>(v));
        else store_pairs<T, E>(dx + units.col(t + i * L), v);
      }
  }
  if (!p.dweight.data && !p.dbias.data) return;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < P; ++j) {
      if (!SHIFT)
#pragma unroll
        for (int o = L; o < 32; o <<= 1) {
          dw[i][j] = add2(dw[i][j], __shfl_xor_sync(0xffffffffu, dw[i][j], o));
          db[i][j] = add2(db[i][j], __shfl_xor_sync(0xffffffffu, db[i][j], o));
        }
      if ((SHIFT || sub == 0) && i < count) {
        const int c = units.col(t + i * L) + 2 * j;
        float* at = s_sums + (SHIFT ? warp * R + sub : warp) * 2 * p.dim + c;
        const float2 a = unpack2(dw[i][j]), b = unpack2(db[i][j]);
        if (!SHIFT || units.in(t + i * L, 2 * j)) at[0] = a.x, at[p.dim] = b.x;
        if (!SHIFT || units.in(t + i * L, 2 * j + 1)) at[1] = a.y, at[p.dim + 1] = b.y;
      }
    }
  __syncthreads();
  const SumsOut out = sums_out(p, g);
  for (int c = threadIdx.x; c < 2 * p.dim; c += blockDim.x) {
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < SETS; ++q) v += s_sums[q * 2 * p.dim + c];
    if (c < p.dim && out.dw) out.dw[c] = v;
    if (c >= p.dim && out.db) out.db[c - p.dim] = v;
  }
}

// 32 columns per block, blockDim.y parts at a time, of dweight's sums (blockIdx.z = 0) or dbias's. Bound: latency (152
// parts of 4096 columns, 5 MB, 6 us).
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

// How a backward call runs: by warps (short rows), through rings (whole units), in units off the 16-byte grid, or
// element by element; its blocks per group, whose sums are parts where there are several.
struct BackPlan {
  enum { SHORT, STREAM, SHIFT, SINGLE } kind;
  StreamShape s;  // (per_sm: teams of a block, one to an SM)
  BackStage stage;
  int blocks;
  int teams() const { return s.per_sm; }
  bool shift;  // SHORT: off the 16-byte grid
};
// Lanes of a row in k_layer_back_short, two vectors to each.
int back_lanes(int64_t nvec) {
  int lanes = 4;
  while (lanes < 32 && lanes * 2 < nvec) lanes *= 2;
  return lanes;
}
// A block of 16 elements per thread (32 where 512 threads do not reach a row's end), and its ring.
StreamShape back_shape(const lipz_layernorm_backward_args& a, BackStage* b) {
  const int eb = type_bytes(a.dy.type), e = 16 / eb, dim = (int)a.dim;
  const int nvec = (int)ceil_div(dim + (back_vec(a) ? 0 : e - 1), e);
  StreamShape s{};
  s.wide = row_threads(nvec, 16 / e) > 512;
  s.tpr = row_threads(nvec, (s.wide ? 32 : 16) / e);
  const int bytes[4] = {dim * eb, a.kept.data ? dim : dim * eb,
                        a.kept.data ? (int)ceil_div(dim, LIPZ_BLOCK) : 0, a.dsum.data ? dim * eb : 0};
  int at = 0;
  for (int i = 0; i < 4; ++i) {
    b->bytes[i] = bytes[i], b->at[i] = at;
    if (bytes[i]) at += (int)ceil_div(bytes[i], 16) * 16 + 32;  // (a unit before the row, and one after)
  }
  s.row = s.slot = at;
  s.share(TEAM_THREADS);
  return s;
}

BackPlan back_plan(const lipz_layernorm_backward_args& a) {
  BackPlan b{};
  const int eb = type_bytes(a.dy.type), e = 16 / eb;
  const int64_t groups = a.groups > 0 ? a.groups : 1;
  auto blocks = [&](int per_sm, int rows) {
    const int64_t fill = (int64_t)per_sm * sm_count() / groups, most = ceil_div(a.rows, rows);
    const int64_t n = fill < most ? fill : most;
    return n < 1 ? 1 : (int)n;
  };
  auto by_warps = [&](int64_t nvec) {
    b.kind = BackPlan::SHORT;
    const int lanes = back_lanes(nvec);
    const int warps = BACK_WARPS, set = warps * 32 / lanes;
    b.blocks = blocks(16 / warps, 2 * set);
    // one block per group needs no second launch: where its turns are few, or more would come one after the other
    const int64_t fill = (int64_t)(16 / warps) * sm_count() / groups;
    if (fill < 4 && (ceil_div(a.rows, set) <= 16 || ceil_div(b.blocks * groups, sm_count()) >= b.blocks)) b.blocks = 1;
    return b;
  };
  if (back_vec(a)) {
    if (a.dim / e <= 64) return by_warps(a.dim / e);
    b.kind = BackPlan::STREAM;
    b.s = back_shape(a, &b.stage);
    b.blocks = blocks(1, 4 * b.teams());
    return b;
  }
  auto same = [&](const lipz_mat& m) { return same_shift(a.dy, m, a.groups, a.rows, e); };
  if (a.dim <= SHIFT_DIM && same(a.dx) && same(a.dsum) && (a.kept.data || same(a.s))) {
    const int64_t units = ceil_div(a.dim + e - 1, e);
    b.shift = true;
    // (a warp's work on a row's ends weighs the more, the fewer rows share it, but rings of many groups leave each few
    // blocks: 131072 x 77 53 us by warps, 95 through rings, 65536 x 301 89 and 71, 144 groups of 100 x 257 21 and 52)
    if (units <= 16 || (units <= 64 && groups >= 8)) return by_warps(units);
    b.kind = BackPlan::SHIFT;
    b.s = back_shape(a, &b.stage);
    b.blocks = (int)shift_blocks(blocks(1, 4 * b.teams()), ceil_div(a.rows, b.teams()), e);
    if (b.blocks < 1) b.blocks = 1;
    return b;
  }
  b.kind = BackPlan::SINGLE;
  b.blocks = blocks(2, 4);
  return b;
}

template <auto KERNEL>
cudaError_t launch_back_rings(const LayerBack& p, const BackPlan& b, int64_t groups, cudaStream_t st) {
  const cudaError_t e = allow_smem<KERNEL>();
  if (e != cudaSuccess) return e;
  const int sums = b.teams() > 1 ? b.teams() * 2 * p.dim * 4 : 0, rings = b.teams() * b.s.smem;
  return launch_pdl(KERNEL, dim3(b.blocks, (unsigned)groups), dim3(b.s.tpr * b.teams()), rings > sums ? rings : sums, st,
                    p, b.stage, b.s.tpr, b.s.stages, b.s.slot, timeout_word());
}
template <typename T, int L, bool KEPT, bool SHIFT>
cudaError_t launch_back_short(const LayerBack& p, int64_t groups, int blocks, cudaStream_t st) {
  constexpr auto kernel = k_layer_back_short<T, 16 / sizeof(T), 2, L, KEPT, SHIFT>;
  const cudaError_t e = allow_smem<kernel>();
  return e != cudaSuccess ? e
                          : launch_pdl(kernel, dim3(blocks, (unsigned)groups), dim3(32 * BACK_WARPS),
                                       (size_t)BACK_WARPS * (SHIFT ? 32 / L : 1) * 2 * p.dim * 4, st, p);
}
template <typename T, bool KEPT, bool SHIFT>
cudaError_t launch_back_short(const LayerBack& p, int64_t groups, int blocks, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  const int lanes = back_lanes(ceil_div(p.dim + (SHIFT ? E - 1 : 0), E));
  if (lanes == 32) return launch_back_short<T, 32, KEPT, SHIFT>(p, groups, blocks, st);
  if (lanes == 16) return launch_back_short<T, 16, KEPT, SHIFT>(p, groups, blocks, st);
  if (lanes == 8) return launch_back_short<T, 8, KEPT, SHIFT>(p, groups, blocks, st);
  return launch_back_short<T, 4, KEPT, SHIFT>(p, groups, blocks, st);
}
template <typename T, bool KEPT>
cudaError_t launch_back(const LayerBack& p, const BackPlan& b, int64_t groups, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  if (b.kind == BackPlan::SHORT)
    return b.shift ? launch_back_short<T, KEPT, true>(p, groups, b.blocks, st)
                   : launch_back_short<T, KEPT, false>(p, groups, b.blocks, st);
  if (b.kind == BackPlan::STREAM)
    return b.s.wide ? launch_back_rings<k_layer_back_stream<T, E, 32 / E, KEPT, false>>(p, b, groups, st)
                    : launch_back_rings<k_layer_back_stream<T, E, 16 / E, KEPT, false>>(p, b, groups, st);
  if (b.kind == BackPlan::SHIFT) return launch_back_rings<k_layer_back_stream<T, E, 16 / E, KEPT, true>>(p, b, groups, st);
  const int nv = row_threads(p.dim, 16) <= 512 ? 16 : 32;
  const dim3 grid(b.blocks, (unsigned)groups), block(row_threads(p.dim, nv));
  return nv == 16 ? launch_pdl(k_layer_backward<T, 16, KEPT>, grid, block, 0, st, p)
                  : launch_pdl(k_layer_backward<T, 32, KEPT>, grid, block, 0, st, p);
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
  auto go = [&] {
    if (a.x.type == LIPZ_FP32) return vec ? launch_layer<float, 4>(p, st) : launch_layer<float, 1>(p, st);
    return vec ? launch_layer<bf16, 8>(p, st) : launch_layer<bf16, 1>(p, st);
  };
  // Rows in units have their checkpoint's blocks across threads: a launch of its own, of x before y may be written
  // over it, or of the sum after.
  if (!a.kept.data || vec || !layer_shift(p)) return go();
  p.kept.data = nullptr;
  lipz_checkpoint_rows_args c{};
  c.groups = a.groups, c.rows = a.rows, c.dim = a.dim, c.x = a.residual.data ? a.sum : a.x, c.c = a.kept;
  cudaError_t e2 = a.residual.data ? go() : checkpoint_rows(c, st);
  if (e2 != cudaSuccess) return e2;
  return a.residual.data ? checkpoint_rows(c, st) : go();
}

namespace {
uint64_t back_space(const lipz_layernorm_backward_args& a, const BackPlan& b) {
  return b.blocks > 1 && (a.dweight.data || a.dbias.data) ? (uint64_t)a.groups * b.blocks * 2 * a.dim * 4 : 0;
}
}  // namespace

uint64_t layernorm_backward_workspace(const lipz_layernorm_backward_args& a) {
  return a.dweight.data || a.dbias.data ? back_space(a, back_plan(a)) : 0;
}

cudaError_t layernorm_backward(const lipz_layernorm_backward_args& a, cudaStream_t st, uint64_t* need) {
  *need = 0;
  if (a.groups == 0) return cudaSuccess;
  const BackPlan b = back_plan(a);
  *need = back_space(a, b);
  if (!space_given(a.workspace, a.workspace_bytes, *need)) return cudaSuccess;
  const bool parts = *need, kept = a.kept.data;
  const LayerBack p{a.dy, a.s, a.dsum, a.dx, a.kept, a.weight, a.mean, a.rstd, a.dweight, a.dbias,
                    parts ? (float*)a.workspace : nullptr, a.rows, (int)a.dim, 1.f / (float)a.dim};
  cudaError_t e;
  if (a.dy.type == LIPZ_FP32)
    e = kept ? launch_back<float, true>(p, b, a.groups, st) : launch_back<float, false>(p, b, a.groups, st);
  else
    e = kept ? launch_back<bf16, true>(p, b, a.groups, st) : launch_back<bf16, false>(p, b, a.groups, st);
  if (e != cudaSuccess || !parts) return e;
  const int ways = b.blocks >= 128 ? 32 : b.blocks >= 16 ? 8 : 1;
  return launch_pdl(k_sum_pairs, dim3((unsigned)ceil_div(a.dim, 32), (unsigned)a.groups, 2), dim3(32, ways), 0, st,
                    p.part, b.blocks, (int64_t)a.dim, a.dweight, a.dbias);
}

}  // namespace ops
}  // namespace lipz
