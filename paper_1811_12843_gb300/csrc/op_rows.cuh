// Device and host helpers of the kernels over rows (op_norm.cu, op_layernorm.cu): sums of a row, 8-bit scales, rings
// of shared-memory stages, rows off the 16-byte grid, and the shapes of blocks.
#pragma once

#include "ops.cuh"
#include "tc_ptx.cuh"

namespace lipz {
namespace ops {

namespace {

// A row's sums: of squares, and the largest magnitude's bits.
struct Sums {
  float ss;
  uint32_t top;
};

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
// ---- rings of shared-memory stages, filled by bulk copies. Whole 16-byte units are copied, from the one that
// holds a row's first byte to the one that holds its last.
constexpr int RING_MAX = 8, RING_BARS = 128;  // stages; bytes before the first

struct Ring {
  uint32_t bars, data;
  int stages, slot, arrays;  // slot: bytes of one array's row in a stage
  volatile int* abort_flag;
  int* code;
};

__device__ __forceinline__ Ring ring_of(uint8_t* smem, int stages, int slot, int arrays) {
  Ring q;
  q.bars = tc::smem_u32(smem);
  q.data = q.bars + RING_BARS;
  q.stages = stages, q.slot = slot, q.arrays = arrays;
  q.abort_flag = reinterpret_cast<volatile int*>(smem + 8 * RING_MAX);
  q.code = reinterpret_cast<int*>(smem + 8 * RING_MAX + 4);
  return q;
}
// One thread, before a barrier of those that use the ring.
__device__ __forceinline__ void ring_set_up(const Ring& q) {
  for (int s = 0; s < q.stages; ++s) tc::mbar_init(q.bars + 8 * s, 1);
  *q.abort_flag = 0;
  *q.code = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ Ring ring_init(uint8_t* smem, int stages, int slot, int arrays) {
  const Ring q = ring_of(smem, stages, slot, arrays);
  if (threadIdx.x == 0) ring_set_up(q);
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

// ---- rows off the 16-byte grid, in the whole units that they touch. Parameters stand in shared memory, one word
// in E + 1 left out, so that lanes E columns apart meet different banks.
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

// ---- host
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
  int row, fixed;  // bytes of a stage, and of what stands beside the ring
  void fit() {
    stages = (RING_SMEM / per_sm - 1024 - RING_BARS - fixed) / row;
    if (stages > RING_MAX) stages = RING_MAX;
    smem = RING_BARS + stages * row + fixed;
  }
  // Blocks of `threads` per SM in all, as many as leave each two stages or more.
  void share(int threads) {
    per_sm = threads / tpr < 24 ? threads / tpr : 24;
    if (per_sm < 1) per_sm = 1;
    for (fit(); per_sm > 1 && stages < 2; fit()) --per_sm;
  }
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
  s.row = s.slot * arrays, s.fixed = fixed;
  s.share(s.wide ? threads / 2 : threads);
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

// Whether, in every row, two matrices begin at the same element of a unit of e elements.
bool same_shift(const lipz_mat& a, const lipz_mat& b, int64_t groups, int64_t rows, int e) {
  if (!b.data) return true;
  auto first = [](const lipz_mat& m) { return (int64_t)((uintptr_t)m.data / type_bytes(m.type)); };
  return (first(a) - first(b)) % e == 0 && (rows == 1 || (a.row - b.row) % e == 0) &&
         (groups == 1 || (a.group - b.group) % e == 0);
}

}  // namespace

}  // namespace ops
}  // namespace lipz
