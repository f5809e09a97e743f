// Device helpers of the residual-block operators: element vectors, 8-bit floats, activations.
#pragma once

#include <cuda_fp8.h>

#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "op_gemm.h"

namespace lipz {
namespace ops {

typedef unsigned char e4m3;

constexpr float SCALE_MIN = 1.17549435082228751e-38f;  // 2^-126

// The larger of two values, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// E elements of one access (1, or 16 bytes of the wider types), in registers as they lie in memory.
template <typename T, int E>
struct Raw {
  static_assert(E == 1 || E * sizeof(T) == 16, "one element or 16 bytes");
  uint32_t w[E == 1 ? 1 : 4];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (E > 1) {
      const uint4 r = *reinterpret_cast<const uint4*>(p);
      w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
    } else if constexpr (sizeof(T) == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const unsigned short*>(p);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : w) v = 0;
  }
  __device__ __forceinline__ void clear(int e) {
    if constexpr (sizeof(T) == 4) w[e] = 0;
    else w[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    return e & 1 ? __uint_as_float(w[e >> 1] & 0xFFFF0000u) : __uint_as_float(w[e >> 1] << 16);
  }
};

template <typename T, int E>
__device__ __forceinline__ void load_vec(const T* p, float* v) {
  Raw<T, E> r;
  r.load(p);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = r.get(e);
}

template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  if constexpr (E == 1) {
    *p = from_f<T>(v[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// fp32 parameters beside E elements of a row.
template <int E>
__device__ __forceinline__ void load_params(const float* p, float* v) {
  if constexpr (E == 1) {
    v[0] = __ldg(p);
  } else {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const float4 r = __ldg(reinterpret_cast<const float4*>(p + i));
      v[i] = r.x, v[i + 1] = r.y, v[i + 2] = r.z, v[i + 3] = r.w;
    }
  }
}

// Host: lets a kernel's launches ask for up to `bytes` of dynamic shared memory, once per device (`done`: the
// devices where that is so).
template <typename K>
cudaError_t allow_dynamic_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && done.load() >> dev & 1) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or((uint64_t)1 << dev);
  return e;
}

// Two values to e4m3, to nearest even; past 448 they saturate, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
template <int E>
__device__ __forceinline__ void store_e4m3(e4m3* p, const float* v) {
  if constexpr (E == 1) {
    *p = (e4m3)(e4m3x2(v[0], 0.f) & 0xFF);
  } else {
    uint32_t w[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i)
      w[i] = e4m3x2(v[4 * i], v[4 * i + 1]) | e4m3x2(v[4 * i + 2], v[4 * i + 3]) << 16;
    if constexpr (E == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
}

// ---- activations: forward, and derivative at the pre-activation
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float LOG2E = 1.44269504088896341f;
// 1 / (1 + e^-v): the hardware's exponential and reciprocal, 2^-22 and 2^-23 of the value, and the rounding of the
// exponent LOG2E v, which weighs |v| 2^-23 where e^-v does (2^-17 at v = -80)
__device__ __forceinline__ float logistic(float v) { return rcp_approx(1.f + ex2_approx(-LOG2E * v)); }
// gelu in its tanh form is u logistic(u (GELU_1 + GELU_3 u^2)): no difference of near values
constexpr float GELU_1 = 1.59576912160573071f, GELU_3 = 0.0713548162726009f;

template <int ACT>
__device__ __forceinline__ float act_value(float u, float slope) {
  if constexpr (ACT == LIPZ_ACT_RELU) return u < 0.f ? 0.f : u;
  if constexpr (ACT == LIPZ_ACT_LRELU) return u > 0.f ? u : slope * u;
  if constexpr (ACT == LIPZ_ACT_TANH) {
    // 1 - 2 / (1 + e^(2|u|)), and below 1/4, where that cancels, the Taylor series through u^9
    const float a = fabsf(u);
    const float t = fmaf(-2.f, rcp_approx(1.f + ex2_approx(2.f * LOG2E * a)), 1.f);
    const float a2 = a * a;
    float q = fmaf(a2, 0.021869488536155203f, -0.053968253968253971f);
    q = fmaf(a2, q, 0.13333333333333333f);
    q = fmaf(a2, q, -0.33333333333333333f);
    return copysignf(a < 0.25f ? a * fmaf(a2, q, 1.f) : t, u);
  }
  if constexpr (ACT == LIPZ_ACT_GELU) return u * logistic(u * fmaf(GELU_3, u * u, GELU_1));
  if constexpr (ACT == LIPZ_ACT_SILU) return u * logistic(u);
  return u;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float u, float slope) {
  if constexpr (ACT == LIPZ_ACT_RELU) return u > 0.f ? 1.f : 0.f;
  if constexpr (ACT == LIPZ_ACT_LRELU) return u > 0.f ? 1.f : slope;
  if constexpr (ACT == LIPZ_ACT_TANH) {
    // 1 - tanh^2 = 4 e / (1 + e)^2 with e = e^(-2|u|)
    const float e = ex2_approx(-2.f * LOG2E * fabsf(u)), r = rcp_approx(1.f + e);
    return 4.f * e * r * r;
  }
  if constexpr (ACT == LIPZ_ACT_GELU) {
    // (u^2 stays finite: beside 1 - g = 0 an infinite one would make the slope of a large finite u NaN)
    const float u2 = fminf(u * u, 1e30f), g = logistic(u * fmaf(GELU_3, u2, GELU_1));
    return g + u * g * (1.f - g) * fmaf(3.f * GELU_3, u2, GELU_1);
  }
  if constexpr (ACT == LIPZ_ACT_SILU) {
    const float g = logistic(u);
    return g * fmaf(u, 1.f - g, 1.f);
  }
  return 1.f;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t both(float a) { return pack2(a, a); }

// act_value of two values, in place. Without EXACT the result is good to 2^-16, for results that are then
// rounded to bf16: tanh takes x - x^3/3 below 1/64, where its other form has lost 2^-17.
template <int ACT, bool EXACT>
__device__ __forceinline__ void act_pair(float& a, float& b, float slope) {
  if constexpr (ACT == LIPZ_ACT_TANH || ACT == LIPZ_ACT_GELU || ACT == LIPZ_ACT_SILU) {
    const uint64_t u = pack2(a, b), one = both(1.f);
    if constexpr (ACT == LIPZ_ACT_TANH) {
      const float aa = fabsf(a), ab = fabsf(b);
      const uint64_t m = pack2(aa, ab), m2 = mul2(m, m);
      const float2 arg = unpack2(mul2(m, both(2.f * LOG2E)));
      const float2 y = unpack2(add2(pack2(ex2_approx(arg.x), ex2_approx(arg.y)), one));
      const float2 t = unpack2(fma2(both(-2.f), pack2(rcp_approx(y.x), rcp_approx(y.y)), one));
      uint64_t q = both(-0.33333333333333333f);
      if constexpr (EXACT) {
        q = fma2(m2, both(0.021869488536155203f), both(-0.053968253968253971f));
        q = fma2(m2, q, both(0.13333333333333333f));
        q = fma2(m2, q, both(-0.33333333333333333f));
      }
      const float2 s = unpack2(mul2(m, fma2(m2, q, one)));
      constexpr float small = EXACT ? 0.25f : 0.015625f;
      a = copysignf(aa < small ? s.x : t.x, a);
      b = copysignf(ab < small ? s.y : t.y, b);
    } else {
      uint64_t v = u;
      if constexpr (ACT == LIPZ_ACT_GELU) v = mul2(u, fma2(both(GELU_3), mul2(u, u), both(GELU_1)));
      const float2 arg = unpack2(mul2(v, both(-LOG2E)));
      const float2 y = unpack2(add2(pack2(ex2_approx(arg.x), ex2_approx(arg.y)), one));
      const float2 r = unpack2(mul2(u, pack2(rcp_approx(y.x), rcp_approx(y.y))));
      a = r.x, b = r.y;
    }
  } else {
    a = act_value<ACT>(a, slope);
    b = act_value<ACT>(b, slope);
  }
}

// Calls f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case LIPZ_ACT_RELU: return f(std::integral_constant<int, LIPZ_ACT_RELU>{});
    case LIPZ_ACT_LRELU: return f(std::integral_constant<int, LIPZ_ACT_LRELU>{});
    case LIPZ_ACT_TANH: return f(std::integral_constant<int, LIPZ_ACT_TANH>{});
    case LIPZ_ACT_GELU: return f(std::integral_constant<int, LIPZ_ACT_GELU>{});
    case LIPZ_ACT_SILU: return f(std::integral_constant<int, LIPZ_ACT_SILU>{});
    default: return f(std::integral_constant<int, LIPZ_ACT_NONE>{});
  }
}

// 16 bytes from any address, the first n of them, then zeros: the aligned words that hold them, shifted.
__device__ __forceinline__ uint4 bytes16(const uint8_t* p, int64_t n) {
  if (n <= 0) return make_uint4(0, 0, 0, 0);
  const int off = (int)((uint64_t)p & 3), left = n < 16 ? (int)n : 16;
  const uint32_t* q = reinterpret_cast<const uint32_t*>(p - off);
  uint32_t w[5], r[4];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = 4 * i < off + left ? __ldg(q + i) : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = __funnelshift_r(w[i], w[i + 1], off * 8);
    const int keep = left - 4 * i;  // bytes of this word
    if (keep < 4) r[i] = keep <= 0 ? 0u : r[i] & ((1u << 8 * keep) - 1u);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// A row's copy in whole 16-byte units (the bytes past its last element are zero), by the 32 lanes of a warp.
__device__ __forceinline__ void copy_row(const RowCopy& p, int64_t r) {
  const int64_t g = r / p.rows;
  const uint8_t* s = p.src + g * p.group + (r - g * p.rows) * p.ld;
  uint4* d = (uint4*)p.dst + r * p.units;
#pragma unroll 2
  for (int64_t u = threadIdx.x & 31; u < p.units; u += 32) d[u] = bytes16(s + u * 16, p.bytes - u * 16);
}
// Block `b` of 256 threads: 8 rows, of one copy after the other.
__device__ __forceinline__ void copy_rows(const CopyJobs& jobs, int64_t b) {
  for (int j = 0; j < jobs.n; ++j) {
    const int64_t blocks = (jobs.c[j].total + COPY_ROWS - 1) / COPY_ROWS;
    if (b < blocks) {
      const int64_t r = b * COPY_ROWS + (threadIdx.x >> 5);
      if (r < jobs.c[j].total) copy_row(jobs.c[j], r);
      return;
    }
    b -= blocks;
  }
}
// The epilogue of element (m, n) of group g, from its sum u.
__device__ __forceinline__ void finish(const Epilogue& e, int64_t g, int64_t m, int64_t n, float u) {
  const float b = e.bias.data ? e.bias.data[g * e.bias.group + n] : 0.f;
  // (one scale after the other, as for many rows: their product may leave fp32's range where the result does not)
  if (e.w_scale.data)
    u = fmaf(u * e.x_scale.data[g * e.x_scale.group + m], e.w_scale.data[g * e.w_scale.group + n], b);
  else
    u += b;
  if (e.pre.data)
    ((bf16*)e.pre.data)[g * e.pre.group + m * e.pre.row + n] = __float2bfloat16_rn(u);
  with_act(e.act, [&](auto act) { u = act_value<decltype(act)::value>(u, e.slope); });
  const int64_t ro = g * e.residual.group + m * e.residual.row + n;
  const int64_t yo = g * e.y.group + m * e.y.row + n;
  if (e.y.type == LIPZ_FP32) {
    if (e.residual.data) u += ((const float*)e.residual.data)[ro];
    ((float*)e.y.data)[yo] = u;
  } else {
    if (e.residual.data) u += __bfloat162float(((const bf16*)e.residual.data)[ro]);
    ((bf16*)e.y.data)[yo] = __float2bfloat16_rn(u);
  }
}

}  // namespace ops
}  // namespace lipz
