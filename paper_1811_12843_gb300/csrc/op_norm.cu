// Root-mean-square norm with the residual's addition (forward and backward) and the row quantiser.
//
// A row's elements are read once and stay in the registers of its threads (multiples of 32 of them, NV
// vectors of E elements each, or a part of a warp) between the row's sums and its results. Few rows are
// loaded by their threads; many short ones by warps that take several at a time; many longer ones stream
// through a ring of shared-memory stages. Bound: HBM; a launch and two memory latencies for a few rows.
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace lipz {
namespace ops {

namespace {

struct RowArgs {
  lipz_mat x, residual, sum, y;
  lipz_vec weight, scale, rstd;
  int64_t rows, total;  // of a group, of all
  int dim, tpr, rpb;    // threads per row, rows per block
  float eps, inv_dim;
};

// A row's sums: of squares, and the largest magnitude's bits (as integers, magnitudes keep their order, with
// infinity above every number and NaN above that).
struct Sums {
  float ss;
  uint32_t top;
};
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <bool SUM, bool MAX>
__device__ __forceinline__ Sums warp_reduce(Sums v) {
  if constexpr (SUM) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v.ss += __shfl_xor_sync(0xffffffffu, v.ss, o);
  }
  if constexpr (MAX) v.top = __reduce_max_sync(0xffffffffu, v.top);
  return v;
}
// Over the `warps` warps of a row from `first` on, after a barrier; s[i]: warp i's.
template <bool SUM, bool MAX>
__device__ __forceinline__ Sums join(const Sums* s, int first, int warps) {
  Sums r = s[first];
  for (int i = 1; i < warps; ++i) {
    const Sums q = s[first + i];
    if constexpr (SUM) r.ss += q.ss;
    if constexpr (MAX) r.top = max(r.top, q.top);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ T* row_of(const lipz_mat& m, int64_t g, int64_t r) {
  return reinterpret_cast<T*>(m.data) + g * m.group + r * m.row;
}

// (rows of all groups stay below 2^31)
__device__ __forceinline__ int64_t group_of(const RowArgs& p, int64_t r) {
  return p.total == p.rows ? 0 : (uint32_t)r / (uint32_t)p.rows;
}

// A row's scale in 8 bits from its largest magnitude: top / 448 or 2^-126. 1/448 is the sum of two floats, and the
// quotient comes out to nearest (sevenths are never near halfway between two) down to 2^-100, where the second
// product begins to lose bits.
__device__ __forceinline__ float scale_of(float top) {
  return max_nan(fmaf(top, 0x1.249248p-9f, top * 0x1.24924ap-33f), SCALE_MIN);
}
// 1 / scale as hi + lo, good to 2^-46 (2^-30 where lo is subnormal), so that v hi + v lo rounds to v / scale: a
// value halfway between two of e4m3's goes to the even one. (scale >= 2^-126 and, finite, below 2^120: hi is a
// normal number. Of an infinite scale hi is 0, and so is lo, which the remainder would make NaN.)
struct Reciprocal {
  float hi, lo;
};
__device__ __forceinline__ Reciprocal reciprocal_of(float scale) {
  const float hi = rcp_approx(scale);
  return {hi, hi == 0.f ? 0.f : hi * fmaf(-hi, scale, 1.f)};
}

// What a row's elements (times the weights) are multiplied by, f, and for 8 bits then by 1 / scale (one after the
// other: their product may be infinite). `first`: this thread writes rstd and scale.
struct RowScale {
  float f;
  Reciprocal inv;
};
template <bool QUANT>
__device__ __forceinline__ RowScale row_scale(const RowArgs& p, int64_t g, int64_t gr, Sums red, bool first) {
  RowScale s{1.f, {1.f, 0.f}};
  if (!QUANT) {
    s.f = rsqrtf(fmaf(red.ss, p.inv_dim, p.eps));
    if (first && p.rstd.data) p.rstd.data[g * p.rstd.group + gr] = s.f;
  }
  if (QUANT || p.scale.data) {
    const float scale = scale_of(__uint_as_float(red.top) * s.f);
    if (first) p.scale.data[g * p.scale.group + gr] = scale;
    s.inv = reciprocal_of(scale);
  }
  return s;
}

// Element by element: v f, v w, and the sums of squares; in bf16 rows, whose instructions bound them, two at a
// time (16384 x 4096 quantiser 35 -> 33 us between events, 38 among other calls, norm 54 -> 51; fp32 rows lose by the
// registers that pairs need, but for the two products with 1 / scale).
template <int E>
__device__ __forceinline__ void scale_by(float* v, float f) {
#pragma unroll
  for (int e = 0; e < E; e += E == 8 ? 2 : 1) {
    if constexpr (E == 8) {
      const float2 r = unpack2(mul2(pack2(v[e], v[e + 1]), both(f)));
      v[e] = r.x, v[e + 1] = r.y;
    } else {
      v[e] *= f;
    }
  }
}
template <int E>
__device__ __forceinline__ void scale_by(float* v, Reciprocal r) {
#pragma unroll
  for (int e = 0; e < E; e += E >= 4 ? 2 : 1) {
    if constexpr (E >= 4) {
      const uint64_t q = pack2(v[e], v[e + 1]);
      const float2 u = unpack2(fma2(q, both(r.hi), mul2(q, both(r.lo))));
      v[e] = u.x, v[e + 1] = u.y;
    } else {
      v[e] = fmaf(v[e], r.hi, v[e] * r.lo);
    }
  }
}
template <int E>
__device__ __forceinline__ void times(float* v, const float* w) {
#pragma unroll
  for (int e = 0; e < E; e += E == 8 ? 2 : 1) {
    if constexpr (E == 8) {
      const float2 r = unpack2(mul2(pack2(v[e], v[e + 1]), pack2(w[e], w[e + 1])));
      v[e] = r.x, v[e + 1] = r.y;
    } else {
      v[e] *= w[e];
    }
  }
}
template <int E>
__device__ __forceinline__ void add_squares(const float* v, float2& ss) {
  if constexpr (E == 8) {
    uint64_t a = pack2(ss.x, ss.y);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const uint64_t q = pack2(v[e], v[e + 1]);
      a = fma2(q, q, a);
    }
    ss = unpack2(a);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) ss.x = fmaf(v[e], v[e], ss.x);
  }
}

// A row's results from its sums and its elements (times the weights).
template <typename T, int E, int NV, bool QUANT>
__device__ __forceinline__ void row_results(const RowArgs& p, int64_t g, int64_t gr, Sums red,
                                            float (&v)[NV][E], int t, int tpr, int nvec) {
  const RowScale f = row_scale<QUANT>(p, g, gr, red, t == 0);
  if (QUANT || p.scale.data) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * tpr < nvec) {
        if (!QUANT) scale_by<E>(v[i], f.f);
        scale_by<E>(v[i], f.inv);
        store_e4m3<E>(row_of<e4m3>(p.y, g, gr) + (t + i * tpr) * E, v[i]);
      }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * tpr < nvec) {
        scale_by<E>(v[i], f.f);
        store_vec<T, E>(row_of<T>(p.y, g, gr) + (t + i * tpr) * E, v[i]);
      }
  }
}

// The norm, or with QUANT only the rows' values to 8 bits.
template <typename T, int E, int NV, bool QUANT>
__global__ void __launch_bounds__(E * NV <= 8 ? 1024 : 512) k_rows(const RowArgs p) {
  __shared__ Sums s_red[32];
  const int sub = threadIdx.x / p.tpr, t = threadIdx.x - sub * p.tpr;
  const int64_t r = (int64_t)blockIdx.x * p.rpb + sub;
  const bool live = r < p.total;
  const int64_t g = live ? group_of(p, r) : 0, gr = live ? r - g * p.rows : 0;
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
  const float* weight = QUANT ? nullptr : p.weight.data + g * p.weight.group;
  float2 ss = make_float2(0.f, 0.f);
  float top = 0.f;
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
    if constexpr (!QUANT) {
      add_squares<E>(v[i], ss);
      if (t + i * p.tpr < nvec) {
        float w[E];
        load_params<E>(weight + (t + i * p.tpr) * E, w);
        times<E>(v[i], w);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
  }
  Sums red{ss.x + ss.y, __float_as_uint(top)};
  red = warp_reduce<!QUANT, true>(red);
  if (p.tpr > 32) {
    if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = red;
    __syncthreads();
    red = join<!QUANT, true>(s_red, sub * (p.tpr >> 5), p.tpr >> 5);
  }
  if (live) row_results<T, E, NV, QUANT>(p, g, gr, red, v, t, p.tpr, nvec);
}

// ---- many short rows: a warp walks over sets of 32 / L rows, L lanes to a row of 32 elements each. The next
// set's loads are in flight while this one is summed and written, and a lane's weights stay in its
// registers. No barrier; and a row's fixed work (sums over lanes, places, scales) is shared by 32 / L rows.
// Bound: HBM. Measured against a block and a ring per row, as in k_rows_stream: bf16 131072 x 256 norm 61
// -> 27 us (134 MB, 0.74 of the copy rate), with residual to 8 bits 78 -> 39 (0.89), quantiser 41 -> 18;
// 262144 x 64 113 -> 17; 65536 x 784 68 -> 48; fp32 131072 x 256 68 -> 43 (0.92). With 32 lanes to each row
// 131072 x 256 took 45 us.
constexpr int SHORT_WARPS = 4;  // of a block

// (bf16 in at most 128 registers, for four blocks per SM: three take 31 us)
template <typename T, int E, int L, bool QUANT>
__global__ void __launch_bounds__(32 * SHORT_WARPS, E == 8 ? 4 : 3) k_rows_short(const RowArgs p) {
  constexpr int NV = 32 / E, R = 32 / L;
  const int lane = threadIdx.x & 31, t = lane % L, sub = lane / L, nvec = p.dim / E;
  const int64_t step = (int64_t)gridDim.x * SHORT_WARPS * R;
  const bool has_res = !QUANT && p.residual.data, want_top = QUANT || p.scale.data;
  pdl_wait();
  Raw<T, E> x[NV], res[NV];
  auto bring = [&](int64_t r) {
    const bool live = r < p.total;
    const int64_t g = live ? group_of(p, r) : 0, gr = r - g * p.rows;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * L;
      x[i].zero();
      if (!QUANT) res[i].zero();
      if (live && c < nvec) {
        x[i].load(row_of<const T>(p.x, g, gr) + c * E);
        if (has_res) res[i].load(row_of<const T>(p.residual, g, gr) + c * E);
      }
    }
  };
  float w[NV][E];
  int64_t w_at = -1;  // where in p.weight w is from
  int64_t r = ((int64_t)blockIdx.x * SHORT_WARPS + (threadIdx.x >> 5)) * R + sub;
  bring(r);
  for (; r - sub < p.total; r += step) {  // (the same turns for all lanes of a warp)
    float v[NV][E];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[i][e] = x[i].get(e);
        if (has_res) v[i][e] += res[i].get(e);
      }
    bring(r + step);
    const bool live = r < p.total;
    const int64_t g = live ? group_of(p, r) : 0, gr = r - g * p.rows;
    float2 ss = make_float2(0.f, 0.f);
    float top = 0.f;
    if constexpr (!QUANT) {
      if (live && p.sum.data)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (t + i * L < nvec) store_vec<T, E>(row_of<T>(p.sum, g, gr) + (t + i * L) * E, v[i]);
      if (g * p.weight.group != w_at) {
        w_at = g * p.weight.group;
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (t + i * L < nvec) load_params<E>(p.weight.data + w_at + (t + i * L) * E, w[i]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * L < nvec) {
          add_squares<E>(v[i], ss);
          times<E>(v[i], w[i]);
        }
    }
    if (want_top)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
    Sums red{ss.x + ss.y, __float_as_uint(top)};
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
      if (!QUANT) red.ss += __shfl_xor_sync(0xffffffffu, red.ss, o);
      if (want_top) red.top = max(red.top, __shfl_xor_sync(0xffffffffu, red.top, o));
    }
    if (live) row_results<T, E, NV, QUANT>(p, g, gr, red, v, t, L, nvec);
  }
}

// ---- many rows: a block of one row's threads walks over rows that arrive in a ring of shared-memory
// stages by bulk copies, so that loads stay in flight while rows are summed and written. Whole 16-byte
// units are copied, from the one that holds a row's first byte to the one that holds its last.
constexpr int RING_MAX = 8, RING_BARS = 128;  // stages; bytes before the first

struct Ring {
  uint32_t bars, data;
  int stages, slot, arrays;  // slot: bytes of one array's row in a stage
  volatile int* abort_flag;
  int* code;
};

__device__ __forceinline__ Ring ring_init(uint8_t* smem, int stages, int slot, int arrays) {
  Ring q;
  q.bars = tc::smem_u32(smem);
  q.data = q.bars + RING_BARS;
  q.stages = stages, q.slot = slot, q.arrays = arrays;
  q.abort_flag = reinterpret_cast<volatile int*>(smem + 8 * RING_MAX);
  q.code = reinterpret_cast<int*>(smem + 8 * RING_MAX + 4);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) tc::mbar_init(q.bars + 8 * s, 1);
    *q.abort_flag = 0;
    *q.code = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  return q;
}
// One thread: the rows at `src` (n of them used) into a stage.
__device__ __forceinline__ void ring_load(const Ring& q, int stage, const char* const* src, int bytes) {
  uint32_t size[3], total = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < q.arrays) {
      const uint64_t a = (uint64_t)src[i];
      size[i] = (uint32_t)(((a + bytes + 15) & ~15ull) - (a & ~15ull));
      total += size[i];
    }
  const uint32_t bar = q.bars + 8 * stage;
  tc::mbar_expect_tx(bar, total);
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < q.arrays)
      asm volatile(
          "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
              q.data + (stage * q.arrays + i) * q.slot),
          "l"((uint64_t)src[i] & ~15ull), "r"(size[i]), "r"(bar)
          : "memory");
}
// A wait that expires leaves what is in the stage as it is; the block runs on without waiting and reports.
__device__ __forceinline__ void ring_wait(const Ring& q, int stage, uint32_t parity) {
  if (!*q.abort_flag) tc::mbar_wait(q.bars + 8 * stage, parity, q.abort_flag, q.code, 1);
}
// Where the row of array i begins in a stage.
__device__ __forceinline__ const char* ring_row(const uint8_t* smem, const Ring& q, int stage, int i,
                                                const void* src) {
  return reinterpret_cast<const char*>(smem) + RING_BARS + (stage * q.arrays + i) * q.slot +
         ((uint64_t)src & 15);
}
__device__ __forceinline__ void ring_done(const Ring& q, int* err) {
  __syncthreads();
  if (*q.abort_flag) {  // copies in flight land before the block leaves
    const unsigned long long t0 = tc::globaltimer();
    while (tc::globaltimer() - t0 < 200000ull) {
    }
    if (threadIdx.x == 0 && err) *reinterpret_cast<volatile int*>(err) = *q.code;
    __syncthreads();
  }
}

// The block's sums, with one barrier; s: [2][16], by turns.
template <bool SUM, bool MAX>
__device__ __forceinline__ Sums block_reduce(Sums v, Sums* s) {
  v = warp_reduce<SUM, MAX>(v);
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (warps == 1) {
    __syncwarp();
    return v;
  }
  if ((threadIdx.x & 31) == 0) s[warp] = v;
  __syncthreads();
  return join<SUM, MAX>(s, 0, warps);
}

template <typename T, int E, int NV, bool QUANT>
__global__ void __launch_bounds__(512) k_rows_stream(const RowArgs p, int stages, int slot, int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Sums s_red[2][16];
  const bool has_res = !QUANT && p.residual.data, want_top = QUANT || p.scale.data;
  const Ring q = ring_init(smem, stages, slot, has_res ? 2 : 1);
  const int t = threadIdx.x, tpr = blockDim.x, nvec = p.dim / E, bytes = p.dim * (int)sizeof(T);
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const int64_t g = group_of(p, r), gr = r - g * p.rows;
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
    const int64_t g = group_of(p, r), gr = r - g * p.rows;
    const float* weight = QUANT ? nullptr : p.weight.data + g * p.weight.group;
    const T* gx = row_of<const T>(p.x, g, gr);
    const T* x = reinterpret_cast<const T*>(ring_row(smem, q, stage, 0, gx));
    const T* res = has_res ? reinterpret_cast<const T*>(
                                 ring_row(smem, q, stage, 1, row_of<const T>(p.residual, g, gr)))
                           : nullptr;
    ring_wait(q, stage, turn & 1);
    float v[NV][E];
    float2 ss = make_float2(0.f, 0.f);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      if (c < nvec) {
        load_vec<T, E>(x + c * E, v[i]);
        if (has_res) {
          float w[E];
          load_vec<T, E>(res + c * E, w);
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] += w[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = 0.f;
      }
    }
    // (fp32 rows' squares here leave their weights' loads together: 16384 x 8192 to 8 bits 144 us below, 131 so)
    if constexpr (!QUANT && E == 4 && NV == 4)
#pragma unroll
      for (int i = 0; i < NV; ++i) add_squares<E>(v[i], ss);
    if (!QUANT && p.sum.data) {
      T* s = row_of<T>(p.sum, g, gr);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * tpr < nvec) store_vec<T, E>(s + (t + i * tpr) * E, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (!QUANT) {
        if constexpr (E != 4 || NV != 4) add_squares<E>(v[i], ss);
        if (t + i * tpr < nvec) {
          float w[E];
          load_params<E>(weight + (t + i * tpr) * E, w);
          times<E>(v[i], w);
        }
      }
      if (want_top)
#pragma unroll
        for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
    }
    Sums red{ss.x + ss.y, __float_as_uint(top)};
    red = block_reduce<!QUANT, true>(red, s_red[turn >> 1 & 1]);
    // (the row is in registers everywhere: its stage takes the row that comes `stages` later)
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.total) load(r + (int64_t)stages * gridDim.x, stage);
    row_results<T, E, NV, QUANT>(p, g, gr, red, v, t, tpr, nvec);
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
}

// ---- rows that start off the 16-byte grid (odd widths), all of a call's matrices at the same place of a
// 16-byte unit in each row: threads take the whole units that a row touches, and the first and the last of
// them in part. Parameters stand in shared memory, one word in E + 1 left out, so that lanes E columns apart
// meet different banks. Bound: instructions (bf16 8192 x 8191 norm 64 us, floor 40, quantiser 39, floor 30). Element
// by element, which matrices at different places of a unit and rows past SHIFT_MAX_DIM still are, 16385 x 4097 with
// residual to 8 bits took 262 us, and 332 backward.
// Where a column's parameter stands, E columns of zeros on either side.
template <int E>
__device__ __forceinline__ int padded(int c) {
  return c + E + (c + E) / E;
}

// Element e of unit c is column c E - m + e; `whole`: all of the unit lies in the row.
template <int E>
struct Unit {
  int col;
  bool live, whole;
  __device__ __forceinline__ Unit(int c, int m, int dim)
      : col(c * E - m), live(c * E - m < dim), whole(c * E >= m && c * E - m + E <= dim) {}
  __device__ __forceinline__ bool in(int e, int dim) const { return whole || (col + e >= 0 && col + e < dim); }
};
template <typename T, int E>
__device__ __forceinline__ void store_unit(T* row, const Unit<E>& u, int dim, const float* v) {
  if (u.whole) {
    store_vec<T, E>(row + u.col, v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (u.in(e, dim)) row[u.col + e] = from_f<T>(v[e]);
  }
}
template <int E>
__device__ __forceinline__ void store_unit_e4m3(e4m3* row, const Unit<E>& u, int dim, const float* v) {
  if (u.whole) {
    store_e4m3<E>(row + u.col, v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (u.in(e, dim)) store_e4m3<1>(row + u.col + e, v + e);
  }
}

template <typename T, int E, int NV, bool QUANT>
__global__ void __launch_bounds__(512) k_rows_shift(const RowArgs p, int stages, int slot, int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Sums s_red[2][16];
  const bool has_res = !QUANT && p.residual.data, one = p.total == p.rows || p.weight.group == 0;
  const bool want_top = QUANT || p.scale.data;
  const Ring q = ring_init(smem, stages, slot, has_res ? 2 : 1);
  float* s_w = reinterpret_cast<float*>(smem + RING_BARS + stages * q.arrays * slot);
  const int t = threadIdx.x, tpr = blockDim.x, dim = p.dim, bytes = dim * (int)sizeof(T);
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const int64_t g = group_of(p, r), gr = r - g * p.rows;
    const char* src[3] = {(const char*)row_of<const T>(p.x, g, gr),
                          has_res ? (const char*)row_of<const T>(p.residual, g, gr) : nullptr, nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.total) load(r, s);
    }
  if (!QUANT && one) {
    for (int c = t - E; c < dim + E; c += tpr)
      s_w[padded<E>(c)] = c >= 0 && c < dim ? p.weight.data[c] : 0.f;
    __syncthreads();
  }
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.total; r += gridDim.x) {
    const int64_t g = group_of(p, r), gr = r - g * p.rows;
    const float* weight = QUANT ? nullptr : p.weight.data + g * p.weight.group;
    const int m = (int)((uint64_t)row_of<const T>(p.x, g, gr) & 15) / (int)sizeof(T);
    const uint8_t* x = smem + RING_BARS + stage * q.arrays * slot;
    ring_wait(q, stage, turn & 1);
    float v[NV][E];
    float ss = 0.f, top = 0.f;
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
        if (!QUANT && p.sum.data) store_unit<T, E>(row_of<T>(p.sum, g, gr), u, dim, v[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Unit<E> u(t + i * tpr, m, dim);
      if constexpr (!QUANT) {
#pragma unroll
        for (int e = 0; e < E; ++e) ss = fmaf(v[i][e], v[i][e], ss);
        if (u.live && one) {
          const float* w = s_w + (t + i * tpr) * (E + 1) + E - m;
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] *= w[e + (e >= m)];
        } else if (u.live) {
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] *= u.in(e, dim) ? __ldg(weight + u.col + e) : 0.f;
        }
      }
      if (want_top)
#pragma unroll
        for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(v[i][e]));
    }
    Sums red{ss, __float_as_uint(top)};
    red = block_reduce<!QUANT, true>(red, s_red[turn >> 1 & 1]);
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.total) load(r + (int64_t)stages * gridDim.x, stage);
    const RowScale f = row_scale<QUANT>(p, g, gr, red, t == 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Unit<E> u(t + i * tpr, m, dim);
      if (!u.live) continue;
      if (!QUANT)
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] *= f.f;
      if (QUANT || p.scale.data) {
        scale_by<E>(v[i], f.inv);
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

// Rows too long for the registers of 1024 threads are read twice, one block per row.
template <typename T, int E>
__global__ void __launch_bounds__(1024) k_quantize_long(const RowArgs p, int64_t dim) {
  __shared__ Sums s_red[32];
  const int64_t r = blockIdx.x, g = group_of(p, r), gr = r - g * p.rows;
  const T* x = row_of<const T>(p.x, g, gr);
  e4m3* y = row_of<e4m3>(p.y, g, gr);
  pdl_wait();
  Sums red{0.f, 0u};
  float v[E];
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < dim / E; c += 1024) {
    load_vec<T, E>(x + c * E, v);
#pragma unroll
    for (int e = 0; e < E; ++e) red.top = max(red.top, magnitude(v[e]));
  }
  red = warp_reduce<false, true>(red);
  if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = red;
  __syncthreads();
  red = join<false, true>(s_red, 0, 32);
  const float scale = scale_of(__uint_as_float(red.top));
  if (threadIdx.x == 0) p.scale.data[g * p.scale.group + gr] = scale;
  const Reciprocal inv = reciprocal_of(scale);
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < dim / E; c += 1024) {
    load_vec<T, E>(x + c * E, v);
    scale_by<E>(v, inv);
    store_e4m3<E>(y + c * E, v);
  }
}

struct BackArgs {
  lipz_mat dy, s, dsum, dx;
  lipz_vec weight, rstd, dweight;
  float* part;  // [groups][clusters, or blocks][dim], or null: those of one are the group's
  int64_t rows;
  int dim;
  float inv_dim;
};

// The sums for dweight of a cluster's blocks (place(c): column c's in shared memory), added by the blocks,
// each for a share of the columns. Every thread of the cluster calls it.
template <typename Place>
__device__ __forceinline__ void join_cluster(const BackArgs& p, int64_t g, const float* s_dw, Place place) {
  __syncwarp();
  tc::cluster_sync_all();
  uint32_t size;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int64_t part = blockIdx.x / size, parts = gridDim.x / size;
  float* out = p.part ? p.part + (g * parts + part) * (int64_t)p.dim : p.dweight.data + g * p.dweight.group;
  for (int c = (int)tc::cluster_ctarank() * (int)blockDim.x + threadIdx.x; c < p.dim; c += size * blockDim.x) {
    const uint32_t at = tc::smem_u32(s_dw + place(c));
    float v = 0.f;
    for (uint32_t i = 0; i < size; ++i) {
      float w;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(tc::mapa_shared(at, i)) : "memory");
      v += w;
    }
    out[c] = v;
  }
  __syncwarp();
  tc::cluster_sync_all();  // no block leaves while its sums are read
}

// A block of one row's threads walks over rows of one group (blockIdx.y), which arrive in a ring; its sums
// for dweight stay in registers, and are added over a cluster of blocks in shared memory.
template <typename T, int E, int NV>
__global__ void __launch_bounds__(512) k_rmsnorm_backward(const BackArgs p, int stages, int slot, int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Sums s_red[2][16];
  const bool has_dsum = p.dsum.data;
  const Ring q = ring_init(smem, stages, slot, has_dsum ? 3 : 2);
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, tpr = blockDim.x, nvec = p.dim / E, bytes = p.dim * (int)sizeof(T);
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const char* src[3] = {(const char*)row_of<const T>(p.dy, g, r), (const char*)row_of<const T>(p.s, g, r),
                          has_dsum ? (const char*)row_of<const T>(p.dsum, g, r) : nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.rows) load(r, s);
    }
  const float* weight = p.weight.data + g * p.weight.group;
  float dw[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) dw[i][e] = 0.f;
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float rstd = p.rstd.data[g * p.rstd.group + r];
    const T* sdy = reinterpret_cast<const T*>(ring_row(smem, q, stage, 0, row_of<const T>(p.dy, g, r)));
    const T* ss = reinterpret_cast<const T*>(ring_row(smem, q, stage, 1, row_of<const T>(p.s, g, r)));
    const T* sds = has_dsum ? reinterpret_cast<const T*>(
                                  ring_row(smem, q, stage, 2, row_of<const T>(p.dsum, g, r)))
                            : nullptr;
    ring_wait(q, stage, turn & 1);
    Raw<T, E> dy[NV], s[NV], ds[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      dy[i].zero(), s[i].zero(), ds[i].zero();
      if (c < nvec) {
        dy[i].load(sdy + c * E);
        s[i].load(ss + c * E);
        if (has_dsum) ds[i].load(sds + c * E);
      }
    }
    float along = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      if (c < nvec) {
        float w[E];
        load_params<E>(weight + c * E, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float m = dy[i].get(e) * s[i].get(e);
          dw[i][e] = fmaf(m, rstd, dw[i][e]);
          along = fmaf(m, w[e], along);
        }
      }
    }
    along = block_reduce<true, false>(Sums{along, 0u}, s_red[turn >> 1 & 1]).ss;
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.rows) load(r + (int64_t)stages * gridDim.x, stage);
    // (rstd^2 by itself may be infinite where the gradient is not)
    const float c2 = rstd * (rstd * (along * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      if (c < nvec) {
        float v[E], w[E];
        load_params<E>(weight + c * E, w);
#pragma unroll
        for (int e = 0; e < E; ++e)
          v[e] = fmaf(rstd, fmaf(-s[i].get(e), c2, dy[i].get(e) * w[e]), ds[i].get(e));
        store_vec<T, E>(dx + c * E, v);
      }
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
  if (!p.dweight.data) return;
  float* s_dw = reinterpret_cast<float*>(smem + RING_BARS);  // over the ring
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (t + i * tpr < nvec)
#pragma unroll
      for (int e = 0; e < E; ++e) s_dw[(t + i * tpr) * E + e] = dw[i][e];
  join_cluster(p, g, s_dw, [](int c) { return c; });
}

// The same for rows off the 16-byte grid (k_rows_shift's units): a column is another thread's in every row,
// so the sums for dweight stand in shared memory, beside the weights. Bound: shared memory and instructions
// (bf16 32768 x 1001 68 us, 0.43 of the copy rate, fp32 77, 0.76; with a check of each column's place 83, 87).
template <typename T, int E, int NV>
__global__ void __launch_bounds__(512) k_rmsnorm_backward_shift(const BackArgs p, int stages, int slot,
                                                                int* err) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Sums s_red[2][16];
  const bool has_dsum = p.dsum.data;
  const Ring q = ring_init(smem, stages, slot, has_dsum ? 3 : 2);
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, tpr = blockDim.x, dim = p.dim, bytes = dim * (int)sizeof(T);
  float* s_w = reinterpret_cast<float*>(smem + RING_BARS + stages * q.arrays * slot);
  float* s_dw = s_w + padded<E>(dim + E);
  pdl_wait();
  auto load = [&](int64_t r, int stage) {
    const char* src[3] = {(const char*)row_of<const T>(p.dy, g, r), (const char*)row_of<const T>(p.s, g, r),
                          has_dsum ? (const char*)row_of<const T>(p.dsum, g, r) : nullptr};
    ring_load(q, stage, src, bytes);
  };
  if (t == 0)
    for (int s = 0; s < stages; ++s) {
      const int64_t r = blockIdx.x + (int64_t)s * gridDim.x;
      if (r < p.rows) load(r, s);
    }
  const float* weight = p.weight.data + g * p.weight.group;
  for (int c = t - E; c < dim + E; c += tpr)
    s_w[padded<E>(c)] = c >= 0 && c < dim ? weight[c] : 0.f, s_dw[padded<E>(c)] = 0.f;
  __syncthreads();
  int stage = 0;
  uint32_t turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float rstd = p.rstd.data[g * p.rstd.group + r];
    const int m = (int)((uint64_t)row_of<const T>(p.s, g, r) & 15) / (int)sizeof(T);
    const uint8_t* rows = smem + RING_BARS + stage * q.arrays * slot;
    ring_wait(q, stage, turn & 1);
    Raw<T, E> dy[NV], s[NV], ds[NV];
    float along = 0.f;
    // (bf16 rows keep the weights for the results; with them fp32 rows' registers leave room for fewer blocks:
    // 16384 x 2049 104 us instead of 74)
    float w[NV][E == 8 ? E : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * tpr;
      const Unit<E> u(c, m, dim);
      dy[i].zero(), s[i].zero(), ds[i].zero();
      if (!u.live) continue;
      dy[i].load(reinterpret_cast<const T*>(rows) + c * E);
      s[i].load(reinterpret_cast<const T*>(rows + slot) + c * E);
      if (has_dsum) ds[i].load(reinterpret_cast<const T*>(rows + 2 * slot) + c * E);
      if (!u.whole)  // (what lies beside the row adds nothing, whatever it is)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!u.in(e, dim)) dy[i].clear(e), s[i].clear(e);
      const int at = c * (E + 1) + E - m;  // padded<E>(c E - m + e) = at + e, and from e = m on one more
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = dy[i].get(e) * s[i].get(e);
        const int here = at + e + (e >= m);
        const float we = s_w[here];
        if constexpr (E == 8) w[i][e] = we;
        s_dw[here] = fmaf(d, rstd, s_dw[here]);
        along = fmaf(d, we, along);
      }
    }
    // (the next row's sums for a column follow after this barrier)
    along = block_reduce<true, false>(Sums{along, 0u}, s_red[turn >> 1 & 1]).ss;
    if (t == 0 && r + (int64_t)stages * gridDim.x < p.rows) load(r + (int64_t)stages * gridDim.x, stage);
    const float c2 = rstd * (rstd * (along * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Unit<E> u(t + i * tpr, m, dim);
      if (!u.live) continue;
      float v[E];
      const float* ws = s_w + (t + i * tpr) * (E + 1) + E - m;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float we = E == 8 ? w[i][E == 8 ? e : 0] : ws[e + (e >= m)];
        v[e] = fmaf(rstd, fmaf(-s[i].get(e), c2, dy[i].get(e) * we), ds[i].get(e));
      }
      store_unit<T, E>(dx, u, dim, v);
    }
    turn ^= 2;
    if (++stage == stages) {
      stage = 0;
      turn ^= 1;
    }
  }
  ring_done(q, err);
  if (p.dweight.data) join_cluster(p, g, s_dw, [](int c) { return padded<E>(c); });
}

// Short rows: L lanes to a row, 32 / L rows to a warp, loaded into registers one set ahead; a block of
// WARPS walks over rows of one group, and its warps' sums for dweight are added in shared memory. (With a
// ring and a block per row, 144 x 100 x 256 took 20 us with the parts' sum, two thirds of it the blocks'
// own set-up; 10 so, between events after a flush of L2, and 7.5 among other calls. With 32 lanes to every row bf16
// 131072 x 256 took 54 us instead of 39, 262144 x 64 77 instead of 23.)
template <int NV>
constexpr int BACK_WARPS = NV <= 2 ? 16 : 8;  // (registers)

template <typename T, int E, int NV, int L>
__global__ void __launch_bounds__(32 * BACK_WARPS<NV>) k_rmsnorm_backward_rows(const BackArgs p) {
  constexpr int WARPS = BACK_WARPS<NV>, R = 32 / L;
  extern __shared__ float s_dw[];  // [WARPS][dim]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane % L, sub = lane / L, nvec = p.dim / E;
  const int64_t g = blockIdx.y, step = (int64_t)gridDim.x * WARPS * R;
  pdl_wait();
  float w[NV][E], dw[NV][E];
  const float* weight = p.weight.data + g * p.weight.group;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * L;
#pragma unroll
    for (int e = 0; e < E; ++e) w[i][e] = dw[i][e] = 0.f;
    if (c < nvec) load_params<E>(weight + c * E, w[i]);
  }
  const bool has_dsum = p.dsum.data;
  Raw<T, E> dy[NV], s[NV], ds[NV];
  float rstd = 0.f;
  auto load = [&](int64_t r) {
    if (r >= p.rows) {  // (a row of zeros adds nothing to the sums)
      rstd = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) dy[i].zero(), s[i].zero();
      return;
    }
    rstd = p.rstd.data[g * p.rstd.group + r];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * L;
      if (c < nvec) {
        dy[i].load(row_of<const T>(p.dy, g, r) + c * E);
        s[i].load(row_of<const T>(p.s, g, r) + c * E);
        if (has_dsum) ds[i].load(row_of<const T>(p.dsum, g, r) + c * E);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) dy[i].zero(), s[i].zero(), ds[i].zero();
  int64_t r = ((int64_t)blockIdx.x * WARPS + warp) * R + sub;
  load(r);
  for (; r - sub < p.rows; r += step) {  // (the same turns for all lanes of a warp)
    Raw<T, E> a[NV], b[NV], c3[NV];
    const float f = rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i) a[i] = dy[i], b[i] = s[i], c3[i] = ds[i];
    load(r + step);
    float along = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float m = a[i].get(e) * b[i].get(e);
        dw[i][e] = fmaf(m, f, dw[i][e]);
        along = fmaf(m, w[i][e], along);
      }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) along += __shfl_xor_sync(0xffffffffu, along, o);
    if (r >= p.rows) continue;
    const float c2 = f * (f * (along * p.inv_dim));
    T* dx = row_of<T>(p.dx, g, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * L;
      if (c < nvec) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
          v[e] = fmaf(f, fmaf(-b[i].get(e), c2, a[i].get(e) * w[i][e]), c3[i].get(e));
        store_vec<T, E>(dx + c * E, v);
      }
    }
  }
  if (!p.dweight.data) return;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int o = L; o < 32; o <<= 1) dw[i][e] += __shfl_xor_sync(0xffffffffu, dw[i][e], o);
      if (sub == 0 && t + i * L < nvec) s_dw[warp * p.dim + (t + i * L) * E + e] = dw[i][e];
    }
  __syncthreads();
  float* out = p.part ? p.part + (g * gridDim.x + blockIdx.x) * (int64_t)p.dim
                      : p.dweight.data + g * p.dweight.group;
  for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < WARPS; ++q) v += s_dw[q * p.dim + c];
    out[c] = v;
  }
}

// 32 columns per block, blockDim.y parts at a time: each thread adds every blockDim.y-th part, then the
// threads of a column their sums.
__global__ void __launch_bounds__(1024)
    k_sum_parts(const float* __restrict__ part, int parts, int64_t cols, lipz_vec out) {
  __shared__ float s[32][33];
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x, g = blockIdx.y;
  pdl_wait();
  float v = 0.f;
  if (c < cols) {
    // (sixteen loads in flight: 608 parts of 4096 columns took 13 us with as many as the compiler chose)
    const float* p = part + g * parts * cols + c;
    for (int i0 = threadIdx.y; i0 < parts; i0 += 16 * blockDim.y) {
      float w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int i = i0 + j * blockDim.y;
        w[j] = i < parts ? __ldg(p + i * cols) : 0.f;
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

constexpr int RING_SMEM = 216 * 1024;  // of an SM, for rings and parameters

int row_threads(int nvec, int nv) { return (int)(ceil_div(ceil_div(nvec, nv), 32) * 32); }

// A streaming kernel's block: 16 elements per thread, 32 where 512 threads of 16 do not reach the row's
// end (at LIPZ_NORM_MAX_DIM they do), and as many blocks per SM as its registers allow (`threads` of 16
// elements, half of them of 32) and as leave each two stages or more. Measured, 2048 threads and two
// stages against 1024 and three: norm of 16384 x 8192 with residual to 8 bits 153 and 162 us, backward of
// 16384 x 8192 163 and 210 us, quantiser of 16384 x 8192 77 and 82 us.
struct StreamShape {
  bool wide;
  int tpr, per_sm, stages, slot, smem;
};
// `params`: fp32 parameters of a column that stand in shared memory (k_rows_shift and its backward, whose
// rows touch up to two units more).
// wide: 32 elements per thread wherever the row is.
StreamShape stream_shape(int dim, int e, int eb, int arrays, int threads, int params = 0, bool wide = false) {
  StreamShape s;
  const int nvec = params ? (int)ceil_div(dim + 2 * e - 2, e) : dim / e;
  const int fixed = params * ((dim + 2 * e) / e + 1) * (e + 1) * 4;  // (padded)
  s.wide = row_threads(nvec, 16 / e) > 512 || wide;
  s.tpr = row_threads(nvec, (s.wide ? 32 : 16) / e);
  s.slot = (int)ceil_div((int64_t)dim * eb, 16) * 16 + 16;
  const int row = s.slot * arrays;
  if (s.wide) threads /= 2;
  s.per_sm = threads / s.tpr < 24 ? threads / s.tpr : 24;
  if (s.per_sm < 1) s.per_sm = 1;
  auto stages = [&] { return (RING_SMEM / s.per_sm - 1024 - RING_BARS - fixed) / row; };
  while (s.per_sm > 1 && stages() < 2) --s.per_sm;
  s.stages = stages() > RING_MAX ? RING_MAX : stages();
  s.smem = RING_BARS + s.stages * row + fixed;
  return s;
}

// Allows a kernel that much shared memory, once per device and whatever the call needs: the default limit counts a
// kernel's own arrays too, and a limit that follows the calls would be lowered under another thread's launch.
template <auto KERNEL>
cudaError_t allow_smem() {
  static std::atomic<uint64_t> done{0};
  return allow_dynamic_smem(KERNEL, RING_SMEM, done);
}

// (512 threads of 32 elements, less the two units more)
constexpr int SHIFT_MAX_DIM = 16384 - 16;
// (two parameters and one stage of three fp32 rows in shared memory)
constexpr int SHIFT_BACK_MAX_DIM = 8192;

// From this many rows per SM on, rows stream through rings or are taken by warps, several to each; fewer are
// loaded by the threads that use them.
constexpr int STREAM_ROWS = 4;

// A kernel's registers per thread, and the blocks of tpr threads that an SM then holds, at most `most`: a grid
// of more has its last blocks run alone (k_rows_shift, fp32 8192 x 4097 51 us instead of 63).
int registers_of(const void* kernel) {
  cudaFuncAttributes f;
  if (cudaFuncGetAttributes(&f, kernel) == cudaSuccess) return f.numRegs;
  cudaGetLastError();
  return 64;
}
int blocks_resident(int registers, int tpr, int most) {
  const int held = 65536 / (((registers * 32 + 255) / 256 * 256) * (tpr / 32));
  return held < 1 ? 1 : held < most ? held : most;
}

template <typename T, int E, int NV, bool QUANT>
cudaError_t launch_stream(const RowArgs& p, const StreamShape& s, cudaStream_t st) {
  constexpr auto kernel = k_rows_stream<T, E, NV, QUANT>;
  const cudaError_t e = allow_smem<kernel>();
  if (e != cudaSuccess) return e;
  static const int registers = registers_of((const void*)kernel);
  const int64_t blocks = (int64_t)blocks_resident(registers, s.tpr, s.per_sm) * sm_count();
  return launch_pdl(kernel, dim3((unsigned)(blocks < p.total ? blocks : p.total)), dim3(s.tpr), s.smem,
                    st, p, s.stages, s.slot, timeout_word());
}

// Whether, in every row, two matrices begin at the same element of a unit of e elements.
bool same_shift(const lipz_mat& a, const lipz_mat& b, int64_t groups, int64_t rows, int e) {
  if (!b.data) return true;
  auto first = [](const lipz_mat& m) { return (int64_t)((uintptr_t)m.data / type_bytes(m.type)); };
  return (first(a) - first(b)) % e == 0 && (rows == 1 || (a.row - b.row) % e == 0) &&
         (groups == 1 || (a.group - b.group) % e == 0);
}

template <typename T, int E, int NV, bool QUANT>
cudaError_t launch_shift_of(const RowArgs& p, const StreamShape& s, cudaStream_t st) {
  constexpr auto kernel = k_rows_shift<T, E, NV, QUANT>;
  static const int registers = registers_of((const void*)kernel);
  const cudaError_t e = allow_smem<kernel>();
  const int64_t blocks = (int64_t)blocks_resident(registers, s.tpr, s.per_sm) * sm_count();
  return e != cudaSuccess ? e
                          : launch_pdl(kernel, dim3((unsigned)(blocks < p.total ? blocks : p.total)),
                                       dim3(s.tpr), s.smem, st, p, s.stages, s.slot, timeout_word());
}

template <typename T, bool QUANT>
cudaError_t launch_shift(const RowArgs& p, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  // bf16 rows in 32 elements per thread where two matrices or one of them in 8 bits keep the loads going: 8192 x
  // 4097 with residual to 8 bits 54 -> 50 us, without (norm) 45 -> 54.
  const bool wide = E == 8 && p.dim > 512 && (QUANT || p.residual.data);
  const StreamShape s = stream_shape(p.dim, E, sizeof(T), !QUANT && p.residual.data ? 2 : 1, 2048, 1, wide);
  return s.wide ? launch_shift_of<T, E, 32 / E, QUANT>(p, s, st) : launch_shift_of<T, E, 16 / E, QUANT>(p, s, st);
}

// (one wave of blocks: with a wave and a half 131072 x 256 took 33 us instead of 27)
template <typename T, int E, int L, bool QUANT>
cudaError_t launch_short(const RowArgs& p, cudaStream_t st) {
  static const int resident = [] {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_rows_short<T, E, L, QUANT>,
                                                                        32 * SHORT_WARPS, 0);
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess && n > 0 ? n : 4;
  }();
  const int64_t most = (int64_t)sm_count() * resident, want = ceil_div(p.total, SHORT_WARPS * (32 / L));
  return launch_pdl(k_rows_short<T, E, L, QUANT>, dim3((unsigned)(want < most ? want : most)),
                    dim3(32 * SHORT_WARPS), 0, st, p);
}

template <typename T, int E, bool QUANT>
cudaError_t launch_rows(RowArgs& p, cudaStream_t st) {
  if constexpr (E > 1) {
    const int lanes = (int)ceil_div(p.dim, 32);
    if (p.total > STREAM_ROWS * sm_count() && lanes <= 32) {
      if (lanes <= 2) return launch_short<T, E, 2, QUANT>(p, st);
      if (lanes <= 4) return launch_short<T, E, 4, QUANT>(p, st);
      if (lanes <= 8) return launch_short<T, E, 8, QUANT>(p, st);
      if (lanes <= 16) return launch_short<T, E, 16, QUANT>(p, st);
      return launch_short<T, E, 32, QUANT>(p, st);
    }
  }
  if (p.total > STREAM_ROWS * sm_count()) {
    constexpr int U = 16 / sizeof(T);
    const int64_t groups = p.total / p.rows;
    if (E == 1 && p.dim <= SHIFT_MAX_DIM && same_shift(p.x, p.y, groups, p.rows, U) &&
        same_shift(p.x, p.residual, groups, p.rows, U) && same_shift(p.x, p.sum, groups, p.rows, U))
      return launch_shift<T, QUANT>(p, st);
    // bf16 rows in 32 elements per thread, since a row's fixed work is each thread's: 16384 x 4096 norm 58
    // -> 52 us, with residual to 8 bits 77 -> 73, quantiser 39 -> 35; fp32 rows lose (85 -> 135 us:
    // registers).
    const StreamShape s = stream_shape(p.dim, E, sizeof(T), !QUANT && p.residual.data ? 2 : 1, 2048, 0, E == 8);
    return s.wide ? launch_stream<T, E, 32 / E, QUANT>(p, s, st)
                  : launch_stream<T, E, 16 / E, QUANT>(p, s, st);
  }
  // as many threads as vectors (of 4 single elements), so that a row takes one load latency
  constexpr int few = E == 1 ? 4 : 1;
  const int nvec = p.dim / E, nv = row_threads(nvec, few) <= 1024 ? few : 32 / E;
  p.tpr = row_threads(nvec, nv);
  p.rpb = p.tpr >= 256 ? 1 : 256 / p.tpr;
  const dim3 grid((unsigned)ceil_div(p.total, p.rpb)), block(p.tpr * p.rpb);
  return nv == few ? launch_pdl(k_rows<T, E, few, QUANT>, grid, block, 0, st, p)
                   : launch_pdl(k_rows<T, E, 32 / E, QUANT>, grid, block, 0, st, p);
}

// Vector elements of a backward call: 16 bytes where every row allows it.
bool backward_vec(const lipz_rmsnorm_backward_args& a) {
  const int e = 16 / type_bytes(a.dy.type);
  auto ok = [&](const lipz_mat& m) { return !m.data || rows_aligned(m, a.groups, a.rows, 16); };
  return a.dim % e == 0 && ok(a.dy) && ok(a.s) && ok(a.dsum) && ok(a.dx) &&
         rows_aligned(a.weight, a.groups, 16);
}

// Lanes of a row in k_rmsnorm_backward_rows, two vectors to each (past 32: four to each of 32).
int back_lanes(int64_t nvec) {
  int lanes = 4;
  while (lanes < 64 && lanes * 2 < nvec) lanes *= 2;
  return lanes;
}

// Whether rows go there: up to 128 whole vectors.
bool backward_short(const lipz_rmsnorm_backward_args& a) {
  return backward_vec(a) && ceil_div(a.dim, 16 / type_bytes(a.dy.type)) <= 128;
}

bool backward_shift(const lipz_rmsnorm_backward_args& a) {
  const int e = 16 / type_bytes(a.dy.type);
  return !backward_vec(a) && a.dim <= SHIFT_BACK_MAX_DIM && same_shift(a.s, a.dy, a.groups, a.rows, e) &&
         same_shift(a.s, a.dsum, a.groups, a.rows, e) && same_shift(a.s, a.dx, a.groups, a.rows, e);
}

StreamShape backward_shape(const lipz_rmsnorm_backward_args& a) {
  const int eb = type_bytes(a.dy.type);
  if (backward_shift(a)) return stream_shape((int)a.dim, 16 / eb, eb, a.dsum.data ? 3 : 2, 1024, 2);
  return stream_shape((int)a.dim, backward_vec(a) ? 16 / eb : 1, eb, a.dsum.data ? 3 : 2, 1024);
}

// A cluster's blocks: two where bf16 rows lie on the grid (8192 x 4096 59 -> 56 us). In clusters of 4 or 8,
// four of them per SM, some blocks found no place in their GPC and ran after the others (72 us instead of 53
// without the parts' sum), and so did blocks of k_rmsnorm_backward_shift in clusters of two (bf16 16385 x 777
// 51 -> 71 us); fp32 gains nothing.
int back_cluster(const lipz_rmsnorm_backward_args& a, const StreamShape& s) {
  return a.dy.type == LIPZ_BF16 && backward_vec(a) && !s.wide && s.per_sm % 2 == 0 ? 2 : 1;
}

// Launch in clusters of `cluster` blocks.
template <auto KERNEL>
cudaError_t launch_clusters(const BackArgs& p, const StreamShape& s, int64_t groups, int blocks, int cluster,
                            cudaStream_t st) {
  const cudaError_t e = allow_smem<KERNEL>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks, (unsigned)groups);
  cfg.blockDim = dim3(s.tpr);
  cfg.dynamicSmemBytes = s.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  if (cluster > 1) {
    cudaLaunchAttribute& c = attr[cfg.numAttrs++];
    c.id = cudaLaunchAttributeClusterDimension;
    c.val.clusterDim.x = cluster;
    c.val.clusterDim.y = c.val.clusterDim.z = 1;
  }
  if (st != nullptr && st != cudaStreamLegacy && st != cudaStreamPerThread) {
    cudaLaunchAttribute& c = attr[cfg.numAttrs++];
    c.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    c.val.programmaticStreamSerializationAllowed = 1;
  }
  return cudaLaunchKernelEx(&cfg, KERNEL, p, s.stages, s.slot, timeout_word());
}

template <typename T>
cudaError_t launch_back_shift(const BackArgs& p, const StreamShape& s, int64_t groups, int blocks,
                              cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  return s.wide ? launch_clusters<k_rmsnorm_backward_shift<T, E, 32 / E>>(p, s, groups, blocks, 1, st)
                : launch_clusters<k_rmsnorm_backward_shift<T, E, 16 / E>>(p, s, groups, blocks, 1, st);
}

template <typename T>
cudaError_t launch_back_rows(const BackArgs& p, int64_t groups, int blocks, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  auto go = [&](auto kernel, int warps) {
    return launch_pdl(kernel, dim3(blocks, (unsigned)groups), dim3(32 * warps),
                      (size_t)warps * p.dim * 4, st, p);
  };
  const int lanes = back_lanes(p.dim / E);
  if (lanes > 32) return go(k_rmsnorm_backward_rows<T, E, 4, 32>, BACK_WARPS<4>);
  if (lanes == 32) return go(k_rmsnorm_backward_rows<T, E, 2, 32>, BACK_WARPS<2>);
  if (lanes == 16) return go(k_rmsnorm_backward_rows<T, E, 2, 16>, BACK_WARPS<2>);
  if (lanes == 8) return go(k_rmsnorm_backward_rows<T, E, 2, 8>, BACK_WARPS<2>);
  return go(k_rmsnorm_backward_rows<T, E, 2, 4>, BACK_WARPS<2>);
}

template <typename T, int E>
cudaError_t launch_back(const BackArgs& p, const StreamShape& s, int64_t groups, int blocks, int parts,
                        cudaStream_t st) {
  const int cluster = blocks / parts;
  return s.wide ? launch_clusters<k_rmsnorm_backward<T, E, 32 / E>>(p, s, groups, blocks, cluster, st)
                : launch_clusters<k_rmsnorm_backward<T, E, 16 / E>>(p, s, groups, blocks, cluster, st);
}

}  // namespace

cudaError_t rmsnorm(const lipz_rmsnorm_args& a, cudaStream_t st) {
  RowArgs p{a.x, a.residual, a.sum, a.y, a.weight, a.scale, a.rstd, a.rows, a.groups * a.rows,
            (int)a.dim, 0, 0, a.eps, 1.f / (float)a.dim};
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
                      int ways, cudaStream_t st) {
  return launch_pdl(k_sum_parts, dim3((unsigned)ceil_div(cols, 32), (unsigned)groups), dim3(32, ways), 0, st,
                    part, parts, cols, out);
}

namespace {
// Blocks per group, and the parts in which their sums come.
struct BackBlocks {
  int blocks, parts;
};
BackBlocks backward_blocks(const lipz_rmsnorm_backward_args& a) {
  const int64_t groups = a.groups > 0 ? a.groups : 1;
  if (backward_short(a)) {
    // Sixteen warps per SM. Where that is fewer than four blocks per group, one block per group, which needs no
    // second launch, while its turns are few (bf16 40 groups of 100 x 256 10 us, by three blocks 13, but 6000 x 256
    // 150 and 72; 60 of 1000 x 256 30 and 24) or more blocks would come one after the other (144 of 1000 x 1024
    // 156, by two 162, but 90 130, by three 109).
    const int lanes = back_lanes(ceil_div(a.dim, 16 / type_bytes(a.dy.type)));
    const int warps = lanes > 32 ? BACK_WARPS<4> : BACK_WARPS<2>, set = warps * (lanes > 32 ? 1 : 32 / lanes);
    const int64_t fill = (int64_t)(16 / warps) * sm_count() / groups, most = ceil_div(a.rows, 2 * set);
    const int64_t b = fill < most ? fill : most;
    const bool one = fill < 4 && (ceil_div(a.rows, set) <= 16 || ceil_div(b * groups, sm_count()) >= b);
    return one || b < 1 ? BackBlocks{1, 1} : BackBlocks{(int)b, (int)b};
  }
  // four rows or more per block, whole clusters where there are that many
  const StreamShape s = backward_shape(a);
  const int cluster = back_cluster(a, s);
  const int64_t fill = (int64_t)s.per_sm * sm_count() / groups, most = ceil_div(a.rows, 4);
  int64_t b = fill < most ? fill : most;
  if (b < 1) b = 1;
  if (b < cluster) return {(int)b, (int)b};
  b -= b % cluster;
  return {(int)b, (int)b / cluster};
}
}  // namespace

int rmsnorm_backward_parts(const lipz_rmsnorm_backward_args& a) { return backward_blocks(a).parts; }

cudaError_t rmsnorm_backward(const lipz_rmsnorm_backward_args& a, cudaStream_t st) {
  if (a.groups == 0) return cudaSuccess;
  const StreamShape s = backward_shape(a);
  const auto [blocks, parts] = backward_blocks(a);
  const BackArgs p{a.dy, a.s, a.dsum, a.dx, a.weight, a.rstd, a.dweight,
                   parts > 1 ? (float*)a.workspace : nullptr, a.rows, (int)a.dim,
                   1.f / (float)a.dim};
  const bool vec = backward_vec(a);
  cudaError_t e;
  if (backward_short(a))
    e = a.dy.type == LIPZ_FP32 ? launch_back_rows<float>(p, a.groups, blocks, st)
                               : launch_back_rows<bf16>(p, a.groups, blocks, st);
  else if (backward_shift(a))
    e = a.dy.type == LIPZ_FP32 ? launch_back_shift<float>(p, s, a.groups, blocks, st)
                               : launch_back_shift<bf16>(p, s, a.groups, blocks, st);
  else if (a.dy.type == LIPZ_FP32)
    e = vec ? launch_back<float, 4>(p, s, a.groups, blocks, parts, st)
            : launch_back<float, 1>(p, s, a.groups, blocks, parts, st);
  else
    e = vec ? launch_back<bf16, 8>(p, s, a.groups, blocks, parts, st)
            : launch_back<bf16, 1>(p, s, a.groups, blocks, parts, st);
  if (e != cudaSuccess || parts == 1 || !a.dweight.data) return e;
  return sum_parts(p.part, a.groups, parts, a.dim, a.dweight, parts >= 128 ? 32 : parts >= 16 ? 8 : 1, st);
}

}  // namespace ops
}  // namespace lipz
