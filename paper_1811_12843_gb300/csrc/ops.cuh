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

// n / d for 0 <= n < 2^31 as a multiplication: with s = ceil(log2 d) and m = ceil(2^(31 + s) / d), n m /
// 2^(31 + s) is above n / d by less than n / (d 2^31) < 1 / d.
struct Divisor {
  uint32_t mul;
  int shift;
  __device__ __forceinline__ int operator()(int n) const {
    return (int)((uint64_t)(uint32_t)n * mul >> shift);
  }
};
inline Divisor divisor(int64_t d) {
  int s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), 31 + s};
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

// ---- checkpoints: 16 columns share a power of two
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// A block's byte, and what its elements are multiplied by, from its largest magnitude's bits (as integers,
// magnitudes keep their order, with infinity above every number and NaN above that). 127.5 is 2^6 times 1 + 127/128:
// from there on 2^16, added to the bits, carries into the exponent. Of a block with an infinity or NaN the multiplier
// is NaN.
struct BlockScale {
  float inv;
  uint32_t byte;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
  const uint32_t byte = max((top + 0x10000u) >> 23, 7u) - 6u;
  if (top >= 0x7F800000u) return {__uint_as_float(0x7FC00000u), 255u};
  return {__uint_as_float((254u - byte) << 23), byte};
}
// A value's multiple of the power of two, to nearest even, in the low byte: 1.5 2^23 + v inv has no fraction bits.
__device__ __forceinline__ uint32_t block_multiple(float v, float inv) {
  return __float_as_uint(fmaf(v, inv, 12582912.f));
}
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// E multiples of 4 or more, in words.
template <int E>
__device__ __forceinline__ void block_multiples(const float* v, float inv, uint32_t* w) {
#pragma unroll
  for (int i = 0; i < E; i += 4) {
    const float2 a = unpack2(fma2(pack2(v[i], v[i + 1]), both(inv), both(12582912.f)));
    const float2 b = unpack2(fma2(pack2(v[i + 2], v[i + 3]), both(inv), both(12582912.f)));
    w[i / 4] = pack_bytes(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
}
// And back: the power of two of a byte (NaN of 255), and a word's four values.
__device__ __forceinline__ float block_unit(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}
// (q + 128 in the low byte of 2^23 is the number 2^23 + 128 + q)
__device__ __forceinline__ void block_values(uint32_t w, float unit, float* v) {
  const uint32_t u = w ^ 0x80808080u;
  const uint64_t off = both(-8388736.f), by = both(unit);
  const float2 a = unpack2(mul2(add2(pack2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440)),
                                           __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7441))), off), by));
  const float2 b = unpack2(mul2(add2(pack2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7442)),
                                           __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7443))), off), by));
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
// Two such values as bf16, which holds them: the upper halves.
__device__ __forceinline__ uint32_t block_pair(float lo, float hi) {
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}

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

// act_slope of two values, operation by operation as there.
template <int ACT>
__device__ __forceinline__ uint64_t act_slope_pair(uint64_t u, float slope) {
  const float2 f = unpack2(u);
  const uint64_t one = both(1.f);
  auto logistic2 = [&](uint64_t v) {
    const float2 arg = unpack2(mul2(both(-LOG2E), v));
    const float2 y = unpack2(add2(one, pack2(ex2_approx(arg.x), ex2_approx(arg.y))));
    return pack2(rcp_approx(y.x), rcp_approx(y.y));
  };
  if constexpr (ACT == LIPZ_ACT_TANH) {
    const float2 arg = unpack2(mul2(both(-2.f * LOG2E), pack2(fabsf(f.x), fabsf(f.y))));
    const uint64_t e = pack2(ex2_approx(arg.x), ex2_approx(arg.y));
    const float2 y = unpack2(add2(one, e));
    const uint64_t r = pack2(rcp_approx(y.x), rcp_approx(y.y));
    return mul2(mul2(mul2(both(4.f), e), r), r);
  } else if constexpr (ACT == LIPZ_ACT_GELU) {
    const float2 sq = unpack2(mul2(u, u));
    const uint64_t u2 = pack2(fminf(sq.x, 1e30f), fminf(sq.y, 1e30f));
    const uint64_t g = logistic2(mul2(u, fma2(both(GELU_3), u2, both(GELU_1))));
    return fma2(mul2(mul2(u, g), fma2(g, both(-1.f), one)), fma2(both(3.f * GELU_3), u2, both(GELU_1)), g);
  } else if constexpr (ACT == LIPZ_ACT_SILU) {
    const uint64_t g = logistic2(u);
    return mul2(g, fma2(u, fma2(g, both(-1.f), one), one));
  } else {
    return pack2(act_slope<ACT>(f.x, slope), act_slope<ACT>(f.y, slope));
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

// 32 bytes at a time where they lie on such a boundary.
template <bool WIDE>
__device__ __forceinline__ void load32(const void* p, uint32_t* w) {
  if constexpr (WIDE) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
  } else {
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
}
template <bool WIDE>
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  if constexpr (WIDE) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// A row's copy in whole 16-byte units (the bytes past its last element are zero), by the 32 lanes of a warp; of a
// checkpoint's row (p.bytes: its columns) the bf16 values that it stands for, 16 at a time, by p.lanes lanes. KEPT: there
// may be such rows. (Kernels that know of none are shorter: over 8-bit operands 1459 x 88 -> 3947 with both in one kernel
// took 26.9 us, so 25.0, 1137 x 3304 -> 2048 24.8 and 22.9.)
template <bool KEPT>
__device__ __forceinline__ void copy_row(const RowCopy& p, int64_t r) {
  const int64_t g = r / p.rows, at = r - g * p.rows;
  const uint8_t* s = p.src + g * p.group + at * p.ld;
  uint4* d = (uint4*)p.dst + r * p.units;
  if (KEPT && p.scale) {
    const uint8_t* scale = p.scale + g * p.scale_group + at * p.scale_ld;
    const bool whole = ((uint64_t)s & 15) == 0, wide = ((uint64_t)d & 31) == 0;
#pragma unroll 4
    for (int64_t u = threadIdx.x & (p.lanes - 1); 2 * u < p.units; u += p.lanes) {
      const bool full = p.bytes - u * 16 >= 16;
      const uint4 q = whole && full ? __ldg((const uint4*)s + u) : bytes16(s + u * 16, p.bytes - u * 16);
      const float unit = block_unit(__ldg(scale + u));
      const uint32_t qq[4] = {q.x, q.y, q.z, q.w};
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[4];
        block_values(qq[i], unit, v);
        w[2 * i] = block_pair(v[0], v[1]), w[2 * i + 1] = block_pair(v[2], v[3]);
      }
      if (!full) {  // (a NaN block's values end with the row)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (u * 16 + i >= p.bytes) w[i / 2] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      }
      if (wide && 2 * u + 1 < p.units) {
        store32<true>(d + 2 * u, w);
      } else {
        d[2 * u] = make_uint4(w[0], w[1], w[2], w[3]);
        if (2 * u + 1 < p.units) d[2 * u + 1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
    return;
  }
#pragma unroll 2
  for (int64_t u = threadIdx.x & 31; u < p.units; u += 32) d[u] = bytes16(s + u * 16, p.bytes - u * 16);
}
// Block `b` of 256 threads: 8 rows per warp's worth of lanes, of one copy after the other.
template <bool KEPT>
__device__ __forceinline__ void copy_rows(const CopyJobs& jobs, int64_t b) {
  for (int j = 0; j < jobs.n; ++j) {
    const int lanes = KEPT ? jobs.c[j].lanes : 32, rows = COPY_ROWS * 32 / lanes;
    const int64_t blocks = (jobs.c[j].total + rows - 1) / rows;
    if (b < blocks) {
      const int64_t r = b * rows + threadIdx.x / lanes;
      if (r < jobs.c[j].total) copy_row<KEPT>(jobs.c[j], r);
      return;
    }
    b -= blocks;
  }
}
// The epilogue of element (m, n) of group g, from its sum: u, and the results from it.
__device__ __forceinline__ float pre_activation(const Epilogue& e, int64_t g, int64_t m, int64_t n, float u) {
  const float b = e.bias.data ? e.bias.data[g * e.bias.group + n] : 0.f;
  // (one scale after the other, as for many rows: their product may leave fp32's range where the result does not)
  if (e.w_scale.data)
    return fmaf(u * e.x_scale.data[g * e.x_scale.group + m], e.w_scale.data[g * e.w_scale.group + n], b);
  return u + b;
}
__device__ __forceinline__ void finish_from(const Epilogue& e, int64_t g, int64_t m, int64_t n, float u) {
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
__device__ __forceinline__ void finish(const Epilogue& e, int64_t g, int64_t m, int64_t n, float u) {
  finish_from(e, g, m, n, pre_activation(e, g, m, n, u));
}
// The same with u kept as a checkpoint, by the 16 lanes of a half-warp that hold a block's columns (live: n is one).
__device__ __forceinline__ void finish_kept(const Epilogue& e, int64_t g, int64_t m, int64_t n, bool live, float u) {
  const int lane = threadIdx.x & 31;
  if (live) u = pre_activation(e, g, m, n, u);
  uint32_t top = live ? magnitude(u) : 0u;
#pragma unroll
  for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFu << (lane & 16), top, o));
  if (!live) return;
  const BlockScale s = block_scale(top);
  e.kept.data[g * e.kept.group + m * e.kept.row + n] = (int8_t)block_multiple(u, s.inv);
  if (lane % 16 == 0) e.kept.scale[g * e.kept.scale_group + m * e.kept.scale_row + (n >> 4)] = (uint8_t)s.byte;
  finish_from(e, g, m, n, u);
}

}  // namespace ops
}  // namespace lipz
