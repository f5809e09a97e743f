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
template <int E>
__device__ __forceinline__ void load_pairs(const float* p, uint64_t* w) {
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
// Of the squares of distances from a mean, over the first `count` vectors.
template <int E, int NV>
__device__ __forceinline__ float pairs_squares(const uint64_t (&v)[NV * E / 2], float mean, int count) {
  uint64_t a = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < count)
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

// ---- many short rows: a warp walks over sets of 32 / L rows, L lanes to a row of NV vectors each. The next set's
// loads are in flight while this one is summed and written; weights and biases stay in a lane's registers where a
// lane has 16 elements. No barrier.
constexpr int SHORT_WARPS = 4;  // of a block

template <typename T, int E, int NV, int L>
__global__ void __launch_bounds__(32 * SHORT_WARPS, E == 4 && NV == 8 ? 3 : 4) k_layer_short(const LayerArgs p) {
  constexpr int R = 32 / L;
  constexpr bool HELD = NV * E <= 16;
  const int lane = threadIdx.x & 31, t = lane % L, sub = lane / L, nvec = p.dim / E;
  const int64_t step = (int64_t)gridDim.x * SHORT_WARPS * R;
  const bool has_res = p.residual.data;
  int count = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) count += t + i * L < nvec;
  pdl_wait();
  Raw<T, E> x[NV], res[NV];
  auto bring = [&](int64_t r) {
    const bool live = r < p.total;
    const int64_t g = live ? group_at(r, p.rows, p.total) : 0, gr = r - g * p.rows;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i].zero(), res[i].zero();
      if (live && i < count) {
        x[i].load(row_of<const T>(p.x, g, gr) + (t + i * L) * E);
        if (has_res) res[i].load(row_of<const T>(p.residual, g, gr) + (t + i * L) * E);
      }
    }
  };
  constexpr int P = E / 2;
  uint64_t w[HELD ? NV * P : P], b[HELD ? NV * P : P];
  int64_t held_of = -1;  // the group whose parameters w and b are
  auto params = [&](int64_t g, int i, int at) {
    const int c = (t + i * L) * E;
#pragma unroll
    for (int j = 0; j < P; ++j) b[at + j] = 0;
    load_pairs<E>(p.weight.data + g * p.weight.group + c, w + at);
    if (p.bias.data) load_pairs<E>(p.bias.data + g * p.bias.group + c, b + at);
  };
  int64_t r = ((int64_t)blockIdx.x * SHORT_WARPS + (threadIdx.x >> 5)) * R + sub;
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
    bring(r + step);
    const bool live = r < p.total;
    const int64_t g = live ? group_at(r, p.rows, p.total) : 0, gr = r - g * p.rows;
    if (p.sum.data || p.kept.data) {
      T* s = p.sum.data ? row_of<T>(p.sum, g, gr) : nullptr;
      int8_t* q = p.kept.data + g * p.kept.group + gr * p.kept.row;
      uint8_t* scale = p.kept.scale + g * p.kept.scale_group + gr * p.kept.scale_row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool here = live && i < count;
        const Raw<T, E> u = rounded<T, E>(v + i * P);
        if (s && here) store_raw<T, E>(s + (t + i * L) * E, u);
        if (p.kept.data) keep_raw<T, E>(q, scale, (t + i * L) * E, here, u);
      }
    }
    float sum = pairs_sum(v);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float mean = sum * p.inv_dim;
    float m2 = pairs_squares<E, NV>(v, mean, count);
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
          top = pairs_affine<E, true>(v + i * P, mo, w + (HELD ? i * P : 0), b + (HELD ? i * P : 0), top);
        }
      uint32_t most = __float_as_uint(top);
#pragma unroll
      for (int o = L / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
      const float scale = scale_of(__uint_as_float(most));
      const Reciprocal inv = reciprocal_of(scale);
      if (!live) continue;
      if (t == 0) p.scale.data[g * p.scale.group + gr] = scale;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) store_pairs_e4m3<E>(row_of<e4m3>(p.y, g, gr) + (t + i * L) * E, v + i * P, inv);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (live && i < count) {
          if (!HELD) params(g, i, 0);
          pairs_affine<E, false>(v + i * P, mo, w + (HELD ? i * P : 0), b + (HELD ? i * P : 0), 0.f);
          store_pairs<T, E>(row_of<T>(p.y, g, gr) + (t + i * L) * E, v + i * P);
        }
    }
  }
}

// ---- many rows: a block of one row's threads walks over rows that arrive in a ring of shared-memory stages by bulk
// copies, so that loads stay in flight while rows are summed and written.
template <typename T, int E, int NV>
__global__ void __launch_bounds__(512, E * NV == 16 || E == 8 ? 2 : 1) k_layer_stream(const LayerArgs p, int stages, int slot, int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float4 s_share[2][16];
  __shared__ uint32_t s_top[2][16];
  const bool has_res = p.residual.data;
  const Ring q = ring_init(smem, stages, slot, has_res ? 2 : 1);
  const int t = threadIdx.x, tpr = blockDim.x, nvec = p.dim / E, bytes = p.dim * (int)sizeof(T);
  const int warp = t >> 5, warps = tpr >> 5;
  int count = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) count += t + i * tpr < nvec;
  const float n = (float)__reduce_add_sync(0xffffffffu, count * E), inv_n = n > 0.f ? 1.f / n : 0.f;
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const int64_t g = group_at(r, p.rows, p.total), gr = r - g * p.rows;
    const char* src[3] = {(const char*)row_of<const T>(p.x, g, gr),
                          has_res ? (const char*)row_of<const T>(p.residual, g, gr) : nullptr, nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.total) load(r, s);
    }
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.total; r += gridDim.x) {
    const int64_t g = group_at(r, p.rows, p.total), gr = r - g * p.rows;
    const T* x = reinterpret_cast<const T*>(ring_row(smem, q, stage, 0, row_of<const T>(p.x, g, gr)));
    const T* res = has_res ? reinterpret_cast<const T*>(
                                 ring_row(smem, q, stage, 1, row_of<const T>(p.residual, g, gr)))
                           : nullptr;
    ring_wait(q, stage, turn & 1);
    constexpr int P = E / 2;
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
    const float sum = warp_sum(pairs_sum(v)), own = sum * inv_n;
    const float m2 = warp_sum(pairs_squares<E, NV>(v, own, count));
    float4* shares = s_share[turn >> 1 & 1];
    if ((t & 31) == 0) shares[warp] = make_float4(n, sum, own, m2);
    __syncthreads();
    // (the row is in registers everywhere: its stage takes the row that comes `stages` later)
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.total) load(r + (int64_t)stages * gridDim.x, stage);
    if (p.sum.data || p.kept.data) {
      T* s = p.sum.data ? row_of<T>(p.sum, g, gr) : nullptr;
      int8_t* kq = p.kept.data + g * p.kept.group + gr * p.kept.row;
      uint8_t* scale = p.kept.scale + g * p.kept.scale_group + gr * p.kept.scale_row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Raw<T, E> u = rounded<T, E>(v + i * P);
        if (s && i < count) store_raw<T, E>(s + (t + i * tpr) * E, u);
        if (p.kept.data) keep_raw<T, E>(kq, scale, (t + i * tpr) * E, i < count, u);
      }
    }
    const Moments mo = join_shares(shares, warps, p.inv_dim, p.eps);
    if (t == 0) {
      if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
      if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
    }
    const float* weight = p.weight.data + g * p.weight.group;
    const float* bias = p.bias.data ? p.bias.data + g * p.bias.group : nullptr;
    auto params = [&](int i, uint64_t* w, uint64_t* b) {
      load_pairs<E>(weight + (t + i * tpr) * E, w);
#pragma unroll
      for (int j = 0; j < P; ++j) b[j] = 0;
      if (bias) load_pairs<E>(bias + (t + i * tpr) * E, b);
    };
    if (p.scale.data) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) {
          uint64_t w[P], b[P];
          params(i, w, b);
          top = pairs_affine<E, true>(v + i * P, mo, w, b, top);
        }
      uint32_t* tops = s_top[turn >> 1 & 1];
      uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
      if ((t & 31) == 0) tops[warp] = most;
      __syncthreads();
      most = __reduce_max_sync(0xffffffffu, tops[min(t & 31, warps - 1)]);
      const float scale = scale_of(__uint_as_float(most));
      const Reciprocal inv = reciprocal_of(scale);
      if (t == 0) p.scale.data[g * p.scale.group + gr] = scale;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) store_pairs_e4m3<E>(row_of<e4m3>(p.y, g, gr) + (t + i * tpr) * E, v + i * P, inv);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < count) {
          uint64_t w[P], b[P];
          params(i, w, b);
          pairs_affine<E, false>(v + i * P, mo, w, b, 0.f);
          store_pairs<T, E>(row_of<T>(p.y, g, gr) + (t + i * tpr) * E, v + i * P);
        }
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
}

// ---- rows that start off the 16-byte grid (odd widths), all of a call's matrices at the same place of a 16-byte unit
// in each row: threads take the whole units that a row touches. Weights and biases stand in shared memory.
template <typename T, int E, int NV>
__global__ void __launch_bounds__(512) k_layer_shift(const LayerArgs p, int stages, int slot, int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float4 s_share[2][16];
  __shared__ uint32_t s_top[2][16];
  const bool has_res = p.residual.data;
  const Ring q = ring_init(smem, stages, slot, has_res ? 2 : 1);
  float* s_w = reinterpret_cast<float*>(smem + RING_BARS + stages * q.arrays * slot);
  const int t = threadIdx.x, tpr = blockDim.x, dim = p.dim, bytes = dim * (int)sizeof(T);
  float* s_b = s_w + padded<E>(dim + E);
  const int warp = t >> 5, warps = tpr >> 5;
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const int64_t g = group_at(r, p.rows, p.total), gr = r - g * p.rows;
    const char* src[3] = {(const char*)row_of<const T>(p.x, g, gr),
                          has_res ? (const char*)row_of<const T>(p.residual, g, gr) : nullptr, nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.total) load(r, s);
    }
  int64_t held_of = -1;  // the group whose parameters stand in shared memory
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.total; r += gridDim.x) {
    const int64_t g = group_at(r, p.rows, p.total), gr = r - g * p.rows;
    if (g != held_of) {
      held_of = g;
      const float* weight = p.weight.data + g * p.weight.group;
      const float* bias = p.bias.data ? p.bias.data + g * p.bias.group : nullptr;
      __syncthreads();
      for (int c = t - E; c < dim + E; c += tpr) {
        const bool in = c >= 0 && c < dim;
        s_w[padded<E>(c)] = in ? weight[c] : 0.f, s_b[padded<E>(c)] = in && bias ? bias[c] : 0.f;
      }
      __syncthreads();
    }
    const int m = (int)((uint64_t)row_of<const T>(p.x, g, gr) & 15) / (int)sizeof(T);
    const uint8_t* x = smem + RING_BARS + stage * q.arrays * slot;
    ring_wait(q, stage, turn & 1);
    float v[NV][E];
    int held = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      const Unit<E> u(c, m, dim);
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = 0.f;
      if (u.live) {
        load_vec<T, E>(reinterpret_cast<const T*>(x) + c * E, v[i]);
        if (has_res) {
          float w[E];
          load_vec<T, E>(reinterpret_cast<const T*>(x + slot) + c * E, w);
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] += w[e];
        }
        if (!u.whole)
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (!u.in(e, dim)) v[i][e] = 0.f;
        held += u.whole ? E : min(u.col + E, dim) - max(u.col, 0);
        if (p.sum.data) store_unit<T, E>(row_of<T>(p.sum, g, gr), u, dim, v[i]);
      }
    }
    const float sum = warp_sum(sum_of<E, NV>(v));
    const float n = (float)__reduce_add_sync(0xffffffffu, held), own = n > 0.f ? sum / n : 0.f;
    float m2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Unit<E> u(t + i * tpr, m, dim);
      if (u.live)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float off = u.in(e, dim) ? v[i][e] - own : 0.f;
          m2 = fmaf(off, off, m2);
        }
    }
    m2 = warp_sum(m2);
    float4* shares = s_share[turn >> 1 & 1];
    if ((t & 31) == 0) shares[warp] = make_float4(n, sum, own, m2);
    __syncthreads();
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.total) load(r + (int64_t)stages * gridDim.x, stage);
    const Moments mo = join_shares(shares, warps, p.inv_dim, p.eps);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr, at = c * (E + 1) + E - m;
      const Unit<E> u(c, m, dim);
      if (!u.live) continue;
      // (beside the row weight and bias are zero, and so is what a non-finite mean does not make NaN)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int here = at + e + (e >= m);
        v[i][e] = fmaf((v[i][e] - mo.mean) * mo.rstd, s_w[here], s_b[here]);
        if (p.scale.data && u.in(e, dim)) top = max_nan(top, fabsf(v[i][e]));
      }
    }
    Reciprocal inv{1.f, 0.f};
    if (p.scale.data) {
      uint32_t* tops = s_top[turn >> 1 & 1];
      uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
      if ((t & 31) == 0) tops[warp] = most;
      __syncthreads();
      for (int i = 0; i < warps; ++i) most = max(most, tops[i]);
      const float scale = scale_of(__uint_as_float(most));
      inv = reciprocal_of(scale);
      if (t == 0) p.scale.data[g * p.scale.group + gr] = scale;
    }
    if (t == 0) {
      if (p.mean.data) p.mean.data[g * p.mean.group + gr] = mo.mean;
      if (p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = mo.rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Unit<E> u(t + i * tpr, m, dim);
      if (!u.live) continue;
      if (p.scale.data) {
        scale_by<E>(v[i], inv);
        store_unit_e4m3<E>(row_of<e4m3>(p.y, g, gr), u, dim, v[i]);
      } else {
        store_unit<T, E>(row_of<T>(p.y, g, gr), u, dim, v[i]);
      }
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
}

// One wave of blocks.
template <typename T, int E, int NV, int L>
cudaError_t launch_short(const LayerArgs& p, cudaStream_t st) {
  static const int resident = [] {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_layer_short<T, E, NV, L>,
                                                                        32 * SHORT_WARPS, 0);
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess && n > 0 ? n : 4;
  }();
  const int64_t most = (int64_t)sm_count() * resident, want = ceil_div(p.total, SHORT_WARPS * (32 / L));
  return launch_pdl(k_layer_short<T, E, NV, L>, dim3((unsigned)(want < most ? want : most)), dim3(32 * SHORT_WARPS),
                    0, st, p);
}

template <auto KERNEL>
cudaError_t launch_rings(const LayerArgs& p, StreamShape s, cudaStream_t st) {
  const cudaError_t e = allow_smem<KERNEL>();
  if (e != cudaSuccess) return e;
  static const int registers = registers_of((const void*)KERNEL);
  s.per_sm = blocks_resident(registers, s.tpr, s.per_sm);
  s.fit();
  const int64_t blocks = (int64_t)s.per_sm * sm_count();
  return launch_pdl(KERNEL, dim3((unsigned)(blocks < p.total ? blocks : p.total)), dim3(s.tpr), s.smem, st, p,
                    s.stages, s.slot, timeout_word());
}

// Whether rows go to k_layer_shift: off the 16-byte grid, at the same place of a unit in all of the matrices.
bool layer_shift(const LayerArgs& p) {
  const int e = 16 / type_bytes(p.x.type);
  const int64_t groups = p.total / p.rows;
  return p.total > STREAM_ROWS * sm_count() && p.dim <= SHIFT_MAX_DIM && same_shift(p.x, p.y, groups, p.rows, e) &&
         same_shift(p.x, p.residual, groups, p.rows, e) && same_shift(p.x, p.sum, groups, p.rows, e);
}

template <typename T, int E>
cudaError_t launch_layer(LayerArgs& p, cudaStream_t st) {
  constexpr int U = 16 / sizeof(T);
  const bool many = p.total > STREAM_ROWS * sm_count();
  const int arrays = p.residual.data ? 2 : 1;
  if constexpr (E > 1) {
    const int lanes = (int)ceil_div(p.dim, 16);
    if (many && lanes <= 64) {
      if (lanes <= 4) return launch_short<T, E, 16 / E, 4>(p, st);
      if (lanes <= 8) return launch_short<T, E, 16 / E, 8>(p, st);
      if (lanes <= 16) return launch_short<T, E, 16 / E, 16>(p, st);
      if (lanes <= 32) return launch_short<T, E, 16 / E, 32>(p, st);
      return launch_short<T, E, 32 / E, 32>(p, st);
    }
    if (many) {
      const StreamShape s = stream_shape(p.dim, E, sizeof(T), arrays, 2048, 0, E == 8);
      return s.wide ? launch_rings<k_layer_stream<T, E, 32 / E>>(p, s, st)
                    : launch_rings<k_layer_stream<T, E, 16 / E>>(p, s, st);
    }
  } else if (layer_shift(p)) {
    const StreamShape s = stream_shape(p.dim, U, sizeof(T), arrays, 2048, 2);
    if (s.stages >= 1)
      return s.wide ? launch_rings<k_layer_shift<T, U, 32 / U>>(p, s, st)
                    : launch_rings<k_layer_shift<T, U, 16 / U>>(p, s, st);
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
// The block's two sums, with one barrier; s: [2][16], by turns.
__device__ __forceinline__ float2 block_pair_sum(float2 v, float2* s) {
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const float w = warp_pair(v.x, v.y);
  if ((threadIdx.x & 15) == 0) (&s[warp].x)[threadIdx.x >> 4 & 1] = w;
  __syncthreads();
  float2 r = s[0];
#pragma unroll 4
  for (int i = 1; i < warps; ++i) {
    const float2 q = s[i];
    r.x += q.x, r.y += q.y;
  }
  return r;
}

// A vector of what was normalised, as it lies in memory: of dy's type, or a checkpoint's multiples and their unit.
template <typename T, int E, bool KEPT>
struct Source {
  Raw<T, E> raw;
  __device__ __forceinline__ void zero() { raw.zero(); }
  __device__ __forceinline__ void get(uint64_t* v) const { pairs_of<T, E>(raw, v); }
};
template <typename T, int E>
struct Source<T, E, true> {
  static_assert(E >= 4, "words");
  uint32_t w[E / 4];
  float unit;
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : w) v = 0;
    unit = 0.f;
  }
  __device__ __forceinline__ void load(const int8_t* q, uint32_t byte) {
    if constexpr (E == 8) {
      const uint2 r = *reinterpret_cast<const uint2*>(q);
      w[0] = r.x ^ 0x80808080u, w[1] = r.y ^ 0x80808080u;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(q) ^ 0x80808080u;
    }
    unit = block_unit(byte);
  }
  __device__ __forceinline__ void get(uint64_t* v) const {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const uint64_t a = pack2(__uint_as_float(__byte_perm(w[i], 0x4B000000u, 0x7440)),
                               __uint_as_float(__byte_perm(w[i], 0x4B000000u, 0x7441)));
      const uint64_t b = pack2(__uint_as_float(__byte_perm(w[i], 0x4B000000u, 0x7442)),
                               __uint_as_float(__byte_perm(w[i], 0x4B000000u, 0x7443)));
      v[2 * i] = mul2(add2(a, both(-8388736.f)), both(unit));
      v[2 * i + 1] = mul2(add2(b, both(-8388736.f)), both(unit));
    }
  }
};

// A vector's terms: of the two sums along the row (g, and g (s - mean)) and of those down the columns.
struct Terms {
  uint64_t along_g = 0, along_x = 0;
  __device__ __forceinline__ float2 sums() const {
    const float2 a = unpack2(along_g), b = unpack2(along_x);
    return make_float2(a.x + a.y, b.x + b.y);
  }
};
template <typename T, int E>
__device__ __forceinline__ void add_terms(Terms& t, const Raw<T, E>& dy, const uint64_t* s, const uint64_t* w,
                                          float mean, float rstd, uint64_t* dw, uint64_t* db) {
  uint64_t d[E / 2];
  pairs_of<T, E>(dy, d);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const uint64_t m = mul2(d[j], add2(s[j], both(-mean)));
    dw[j] = fma2(m, both(rstd), dw[j]);
    db[j] = add2(d[j], db[j]);
    t.along_g = fma2(d[j], w[j], t.along_g);
    t.along_x = fma2(m, w[j], t.along_x);
  }
}
// dx = rstd (g - c1 - (s - mean) c2) + dsum
template <typename T, int E>
__device__ __forceinline__ void store_gradient(T* dx, const Raw<T, E>& dy, const uint64_t* s, const uint64_t* w,
                                               const Raw<T, E>& ds, float mean, float rstd, float c1, float c2) {
  uint64_t d[E / 2], v[E / 2];
  pairs_of<T, E>(dy, d);
  pairs_of<T, E>(ds, v);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    const uint64_t a = fma2(add2(s[j], both(-mean)), both(-c2), fma2(d[j], w[j], both(-c1)));
    v[j] = fma2(both(rstd), a, v[j]);
  }
  store_pairs<T, E>(dx, v);
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

// A block of one row's threads walks over rows of one group (blockIdx.y), which arrive in a ring; its sums for dweight
// and dbias stay in registers.
template <typename T, int E, int NV, bool KEPT>
__global__ void __launch_bounds__(512) k_layer_back_stream(const LayerBack p, const BackStage b, int stages, int slot,
                                                           int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float2 s_red[2][16];
  constexpr int P = E / 2;
  const bool has_dsum = p.dsum.data;
  const Ring q = ring_init(smem, stages, slot, 1);
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, tpr = blockDim.x, nvec = p.dim / E;
  int count = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) count += t + i * tpr < nvec;
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const void* src[4];
    back_rows<T, KEPT>(p, g, r, src);
    load_stage(q, b, stage, src);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.rows) load(r, s);
    }
  const float* weight = p.weight.data + g * p.weight.group;
  uint64_t dw[NV][P], db[NV][P];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < P; ++j) dw[i][j] = db[i][j] = 0;
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float mean = p.mean.data[g * p.mean.group + r], rstd = p.rstd.data[g * p.rstd.group + r];
    const void* src[4];
    back_rows<T, KEPT>(p, g, r, src);
    const uint8_t* rows[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) rows[i] = smem + RING_BARS + stage * slot + b.at[i] + ((uint64_t)src[i] & 15);
    ring_wait(q, stage, turn & 1);
    Raw<T, E> dy[NV], ds[NV];
    Source<T, E, KEPT> x[NV];
    Terms terms;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * tpr) * E;
      dy[i].zero(), x[i].zero(), ds[i].zero();
      if (i < count) {
        dy[i].load(reinterpret_cast<const T*>(rows[0]) + c);
        if constexpr (KEPT) x[i].load(reinterpret_cast<const int8_t*>(rows[1]) + c, rows[2][c / LIPZ_BLOCK]);
        else x[i].raw.load(reinterpret_cast<const T*>(rows[1]) + c);
        if (has_dsum) ds[i].load(reinterpret_cast<const T*>(rows[3]) + c);
        uint64_t w[P], s[P];
        load_pairs<E>(weight + c, w);
        x[i].get(s);
        add_terms<T, E>(terms, dy[i], s, w, mean, rstd, dw[i], db[i]);
      }
    }
    const float2 along = block_pair_sum(terms.sums(), s_red[turn >> 1 & 1]);
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.rows) load(r + (int64_t)stages * gridDim.x, stage);
    // (rstd^2 by itself may be infinite where the gradient is not)
    const float c1 = along.x * p.inv_dim, c2 = rstd * (rstd * (along.y * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < count) {
        const int c = (t + i * tpr) * E;
        uint64_t w[P], s[P];
        load_pairs<E>(weight + c, w);
        x[i].get(s);
        store_gradient<T, E>(dx + c, dy[i], s, w, ds[i], mean, rstd, c1, c2);
      }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
  const SumsOut out = sums_out(p, g);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < count)
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int c = (t + i * tpr) * E + 2 * j;
        const float2 a = unpack2(dw[i][j]), b = unpack2(db[i][j]);
        if (out.dw) out.dw[c] = a.x, out.dw[c + 1] = a.y;
        if (out.db) out.db[c] = b.x, out.db[c + 1] = b.y;
      }
}

// Rows off the 16-byte grid, in the units of dy: a column is another thread's in every row, so its sums stand in
// shared memory, beside the weights. A checkpoint's row lies at any byte: its multiples come from the words that hold
// them, and a unit's columns from two blocks at most.
template <typename T, int E, int NV, bool KEPT>
__global__ void __launch_bounds__(512) k_layer_back_shift(const LayerBack p, const BackStage b, int stages, int slot,
                                                          int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float2 s_red[2][16];
  const bool has_dsum = p.dsum.data;
  const Ring q = ring_init(smem, stages, slot, 1);
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, tpr = blockDim.x, dim = p.dim;
  float* s_w = reinterpret_cast<float*>(smem + RING_BARS + stages * slot);
  float *s_dw = s_w + padded<E>(dim + E), *s_db = s_dw + padded<E>(dim + E);
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const void* src[4];
    back_rows<T, KEPT>(p, g, r, src);
    load_stage(q, b, stage, src);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.rows) load(r, s);
    }
  const float* weight = p.weight.data + g * p.weight.group;
  for (int c = t - E; c < dim + E; c += tpr) {
    const int at = padded<E>(c);
    s_w[at] = c >= 0 && c < dim ? weight[c] : 0.f, s_dw[at] = s_db[at] = 0.f;
  }
  __syncthreads();
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float mean = p.mean.data[g * p.mean.group + r], rstd = p.rstd.data[g * p.rstd.group + r];
    const void* src[4];
    back_rows<T, KEPT>(p, g, r, src);
    const int m = (int)((uint64_t)src[0] & 15) / (int)sizeof(T);
    const uint8_t* rows = smem + RING_BARS + stage * slot;
    const uint8_t* scales = rows + b.at[2] + ((uint64_t)src[2] & 15);
    ring_wait(q, stage, turn & 1);
    Raw<T, E> dy[NV], ds[NV];
    float x[NV][E];  // s - mean
    float2 along = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      const Unit<E> u(c, m, dim);
      dy[i].zero(), ds[i].zero();
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] = 0.f;
      if (!u.live) continue;
      dy[i].load(reinterpret_cast<const T*>(rows + b.at[0]) + c * E);
      if (has_dsum) ds[i].load(reinterpret_cast<const T*>(rows + b.at[3]) + c * E);
      if constexpr (KEPT) {
        // (before the row's first column there are up to E - 1 bytes; its slot leaves room for them)
        const int from = b.at[1] + (int)((uint64_t)src[1] & 15) + u.col, off = from & 3;
        const uint32_t* words = reinterpret_cast<const uint32_t*>(rows + (from - off));
        uint32_t w[E / 4 + 1];
#pragma unroll
        for (int j = 0; j <= E / 4; ++j) w[j] = words[j];
        const int first = max(u.col, 0) / LIPZ_BLOCK, last = min(u.col + E - 1, dim - 1) / LIPZ_BLOCK;
        const float unit0 = block_unit(scales[first]), unit1 = block_unit(scales[last]);
        float one[E];
#pragma unroll
        for (int j = 0; j < E / 4; ++j) block_values(__funnelshift_r(w[j], w[j + 1], off * 8), 1.f, one + 4 * j);
#pragma unroll
        for (int e = 0; e < E; ++e)
          x[i][e] = one[e] * ((u.col + e) / LIPZ_BLOCK == first || u.col + e < 0 ? unit0 : unit1);
      } else {
        load_vec<T, E>(reinterpret_cast<const T*>(rows + b.at[1]) + c * E, x[i]);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] -= mean;
      if (!u.whole)  // (what lies beside the row adds nothing, whatever it is)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!u.in(e, dim)) dy[i].clear(e), x[i][e] = 0.f;
      const int at = c * (E + 1) + E - m;  // padded<E>(c E - m + e) = at + e, and from e = m on one more
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int here = at + e + (e >= m);
        const float d = dy[i].get(e), xd = d * x[i][e], we = s_w[here];
        s_dw[here] = fmaf(xd, rstd, s_dw[here]);
        s_db[here] += d;
        along.x = fmaf(d, we, along.x);
        along.y = fmaf(xd, we, along.y);
      }
    }
    // (the next row's sums for a column follow after this barrier)
    along = block_pair_sum(along, s_red[turn >> 1 & 1]);
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.rows) load(r + (int64_t)stages * gridDim.x, stage);
    const float c1 = along.x * p.inv_dim, c2 = rstd * (rstd * (along.y * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr, at = c * (E + 1) + E - m;
      const Unit<E> u(c, m, dim);
      if (!u.live) continue;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e)
        v[e] = fmaf(rstd, fmaf(-x[i][e], c2, fmaf(dy[i].get(e), s_w[at + e + (e >= m)], -c1)), ds[i].get(e));
      store_unit<T, E>(dx, u, dim, v);
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
  const SumsOut out = sums_out(p, g);
  for (int c = t; c < dim; c += tpr) {
    if (out.dw) out.dw[c] = s_dw[padded<E>(c)];
    if (out.db) out.db[c] = s_db[padded<E>(c)];
  }
}

// Short rows: L lanes to a row, 32 / L rows to a warp, loaded into registers one set ahead; a block of WARPS walks over
// rows of one group, and its warps' sums are added in shared memory.
template <int NV>
constexpr int BACK_WARPS = NV <= 2 ? 16 : 8;  // (registers)

template <typename T, int E, int NV, int L, bool KEPT>
__global__ void __launch_bounds__(32 * BACK_WARPS<NV>) k_layer_back_short(const LayerBack p) {
  constexpr int WARPS = BACK_WARPS<NV>, R = 32 / L;
  extern __shared__ float s_sums[];  // [WARPS][2][dim]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane % L, sub = lane / L, nvec = p.dim / E;
  const int64_t g = blockIdx.y, step = (int64_t)gridDim.x * WARPS * R;
  int count = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) count += t + i * L < nvec;
  pdl_wait();
  constexpr int P = E / 2;
  uint64_t w[NV][P], dw[NV][P], db[NV][P];
  const float* weight = p.weight.data + g * p.weight.group;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < P; ++j) w[i][j] = dw[i][j] = db[i][j] = 0;
    if (i < count) load_pairs<E>(weight + (t + i * L) * E, w[i]);
  }
  const bool has_dsum = p.dsum.data;
  Raw<T, E> dy[NV], ds[NV];
  Source<T, E, KEPT> x[NV];
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
        const int c = (t + i * L) * E;
        dy[i].load(row_of<const T>(p.dy, g, r) + c);
        if constexpr (KEPT)
          x[i].load(p.kept.data + g * p.kept.group + r * p.kept.row + c,
                    p.kept.scale[g * p.kept.scale_group + r * p.kept.scale_row + c / LIPZ_BLOCK]);
        else
          x[i].raw.load(row_of<const T>(p.s, g, r) + c);
        if (has_dsum) ds[i].load(row_of<const T>(p.dsum, g, r) + c);
      }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) dy[i].zero(), x[i].zero(), ds[i].zero();
  int64_t r = ((int64_t)blockIdx.x * WARPS + warp) * R + sub;
  load(r);
  for (; r - sub < p.rows; r += step) {  // (the same turns for all lanes of a warp)
    Raw<T, E> a[NV], c3[NV];
    Source<T, E, KEPT> y[NV];
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
        add_terms<T, E>(terms, a[i], s, w[i], m, f, dw[i], db[i]);
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
        uint64_t s[P];
        y[i].get(s);
        store_gradient<T, E>(dx + (t + i * L) * E, a[i], s, w[i], c3[i], m, f, c1, c2);
      }
  }
  if (!p.dweight.data && !p.dbias.data) return;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < P; ++j) {
#pragma unroll
      for (int o = L; o < 32; o <<= 1) {
        dw[i][j] = add2(dw[i][j], __shfl_xor_sync(0xffffffffu, dw[i][j], o));
        db[i][j] = add2(db[i][j], __shfl_xor_sync(0xffffffffu, db[i][j], o));
      }
      if (sub == 0 && i < count) {
        float* at = s_sums + warp * 2 * p.dim + (t + i * L) * E + 2 * j;
        const float2 a = unpack2(dw[i][j]), b = unpack2(db[i][j]);
        at[0] = a.x, at[1] = a.y, at[p.dim] = b.x, at[p.dim + 1] = b.y;
      }
    }
  __syncthreads();
  const SumsOut out = sums_out(p, g);
  for (int c = threadIdx.x; c < 2 * p.dim; c += blockDim.x) {
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < WARPS; ++q) v += s_sums[q * 2 * p.dim + c];
    if (c < p.dim && out.dw) out.dw[c] = v;
    if (c >= p.dim && out.db) out.db[c - p.dim] = v;
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

// How a backward call runs: by warps (short rows), through rings (whole units), in units off the 16-byte grid, or
// element by element; its blocks per group, whose sums are parts where there are several.
struct BackPlan {
  enum { SHORT, STREAM, SHIFT, SINGLE } kind;
  StreamShape s;
  BackStage stage;
  int blocks;
};
// Lanes of a row in k_layer_back_short, two vectors to each (past 32: four to each of 32).
int back_lanes(int64_t nvec) {
  int lanes = 4;
  while (lanes < 64 && lanes * 2 < nvec) lanes *= 2;
  return lanes;
}
// A block of 16 elements per thread (32 where 512 threads do not reach a row's end), and its ring.
StreamShape back_shape(const lipz_layernorm_backward_args& a, int params, BackStage* b) {
  const int eb = type_bytes(a.dy.type), e = 16 / eb, dim = (int)a.dim;
  const int nvec = params ? (int)ceil_div(dim + 2 * e - 2, e) : dim / e;
  StreamShape s{};
  s.wide = row_threads(nvec, 16 / e) > 512;
  s.tpr = row_threads(nvec, (s.wide ? 32 : 16) / e);
  s.fixed = params * ((dim + 2 * e) / e + 1) * (e + 1) * 4;  // (padded)
  const int bytes[4] = {dim * eb, a.kept.data ? dim : dim * eb,
                        a.kept.data ? (int)ceil_div(dim, LIPZ_BLOCK) : 0, a.dsum.data ? dim * eb : 0};
  int at = 0;
  for (int i = 0; i < 4; ++i) {
    b->bytes[i] = bytes[i], b->at[i] = at;
    if (bytes[i]) at += (int)ceil_div(bytes[i], 16) * 16 + 32;  // (a unit before the row, and one after)
  }
  s.row = s.slot = at;
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
  if (back_vec(a)) {
    const int64_t nvec = a.dim / e;
    if (nvec <= 128) {
      b.kind = BackPlan::SHORT;
      const int lanes = back_lanes(nvec);
      const int warps = lanes > 32 ? BACK_WARPS<4> : BACK_WARPS<2>, set = warps * (lanes > 32 ? 1 : 32 / lanes);
      b.blocks = blocks(16 / warps, 2 * set);
      // one block per group needs no second launch: where its turns are few, or more would come one after the other
      const int64_t fill = (int64_t)(16 / warps) * sm_count() / groups;
      if (fill < 4 && (ceil_div(a.rows, set) <= 16 || ceil_div(b.blocks * groups, sm_count()) >= b.blocks)) b.blocks = 1;
      return b;
    }
    b.kind = BackPlan::STREAM;
    b.s = back_shape(a, 0, &b.stage);
    b.s.share(b.s.wide ? 512 : 640);
    b.blocks = blocks(b.s.per_sm, 4);
    return b;
  }
  auto same = [&](const lipz_mat& m) { return same_shift(a.dy, m, a.groups, a.rows, e); };
  if (same(a.dx) && same(a.dsum) && (a.kept.data || same(a.s))) {
    b.s = back_shape(a, 3, &b.stage);
    b.s.share(1024);
    if (b.s.stages >= 1) {
      b.kind = BackPlan::SHIFT;
      b.blocks = blocks(b.s.per_sm, 4);
      return b;
    }
  }
  b.kind = BackPlan::SINGLE;
  b.blocks = blocks(2, 4);
  return b;
}

template <auto KERNEL>
cudaError_t launch_back_rings(const LayerBack& p, const BackPlan& b, int64_t groups, cudaStream_t st) {
  const cudaError_t e = allow_smem<KERNEL>();
  return e != cudaSuccess ? e
                          : launch_pdl(KERNEL, dim3(b.blocks, (unsigned)groups), dim3(b.s.tpr), b.s.smem, st, p,
                                       b.stage, b.s.stages, b.s.slot, timeout_word());
}
template <typename T, int E, int NV, int L, bool KEPT>
cudaError_t launch_back_short(const LayerBack& p, int64_t groups, int blocks, cudaStream_t st) {
  constexpr auto kernel = k_layer_back_short<T, E, NV, L, KEPT>;
  const cudaError_t e = allow_smem<kernel>();
  return e != cudaSuccess ? e
                          : launch_pdl(kernel, dim3(blocks, (unsigned)groups), dim3(32 * BACK_WARPS<NV>),
                                       (size_t)BACK_WARPS<NV> * 2 * p.dim * 4, st, p);
}
template <typename T, bool KEPT>
cudaError_t launch_back(const LayerBack& p, const BackPlan& b, int64_t groups, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  if (b.kind == BackPlan::SHORT) {
    const int lanes = back_lanes(p.dim / E);
    if (lanes > 32) return launch_back_short<T, E, 4, 32, KEPT>(p, groups, b.blocks, st);
    if (lanes == 32) return launch_back_short<T, E, 2, 32, KEPT>(p, groups, b.blocks, st);
    if (lanes == 16) return launch_back_short<T, E, 2, 16, KEPT>(p, groups, b.blocks, st);
    if (lanes == 8) return launch_back_short<T, E, 2, 8, KEPT>(p, groups, b.blocks, st);
    return launch_back_short<T, E, 2, 4, KEPT>(p, groups, b.blocks, st);
  }
  if (b.kind == BackPlan::STREAM)
    return b.s.wide ? launch_back_rings<k_layer_back_stream<T, E, 32 / E, KEPT>>(p, b, groups, st)
                    : launch_back_rings<k_layer_back_stream<T, E, 16 / E, KEPT>>(p, b, groups, st);
  if (b.kind == BackPlan::SHIFT)
    return b.s.wide ? launch_back_rings<k_layer_back_shift<T, E, 32 / E, KEPT>>(p, b, groups, st)
                    : launch_back_rings<k_layer_back_shift<T, E, 16 / E, KEPT>>(p, b, groups, st);
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

uint64_t layernorm_backward_workspace(const lipz_layernorm_backward_args& a) {
  if (!a.dweight.data && !a.dbias.data) return 0;
  const int blocks = back_plan(a).blocks;
  return blocks > 1 ? (uint64_t)a.groups * blocks * 2 * a.dim * 4 : 0;
}

cudaError_t layernorm_backward(const lipz_layernorm_backward_args& a, cudaStream_t st) {
  if (a.groups == 0) return cudaSuccess;
  const BackPlan b = back_plan(a);
  const bool parts = b.blocks > 1 && (a.dweight.data || a.dbias.data), kept = a.kept.data;
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
