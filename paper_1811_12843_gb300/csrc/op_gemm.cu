// Tensor-core product of the residual-block operators (tcgen05, sm_103a):
//     u = (A B^T) x_scale w_scale + bias,   y = act(u) + residual
//
// A tile of C is BM x BN: 128 rows on one CTA, or 256 on a pair of CTAs whose MMAs take A's rows from both
// and half of B's rows from each (so that a byte of B that is brought from L2 serves 256 rows). Persistent
// CTAs walk over tiles and parts of k. Two warps issue the TMA loads of A and of B into a ring of
// 128-byte-swizzled stages, one issues the MMAs into two or four accumulators in tensor memory, one brings
// the tiles' parameters (and residuals) ahead, and sixteen turn accumulators into results.
//
// Bound, and measured (a copy runs at 6.79 TB/s, cuBLAS at 1.94 PFLOP/s in bf16):
//   large k   the tensor cores: backward products of 8192 x 4096 -> 4096 300 us, 1.83 PFLOP/s (0.95);
//             8192 x 4096 -> 8192 over 8-bit operands 174 us by itself (3.2 PFLOP/s), 203 in a row, where the
//             power limit lowers the clock.
//   small k   the way of operands and results through L2: 144 x 500 x 256 -> 784 47 us (208 MB: 31 us).
//   few rows  HBM and latency: 16 x 8192 -> 8192 37 us (134 MB: 20 us), 37 x 1000 -> 500 7.5 us.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <string.h>

#include <type_traits>

#include "op_gemm.h"
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace lipz {
namespace ops {

namespace {

constexpr int ROW = 128;                  // bytes of a swizzled row: 64 bf16 or 128 e4m3 of k
constexpr int EPI_WARPS = 16, FIRST_EPI = 4, THREADS = 32 * (FIRST_EPI + EPI_WARPS);
constexpr int TURN = 32 * 17 * 4;         // a warp's block for turning rows into columns
constexpr int MN_BOX = 64 * ROW;          // 64 k by 64 m (or n) of an operand whose rows run along m (n)
static_assert(EPI_WARPS == SUM_WAYS, "a result warp per way");
// Tensor-core additions truncate: a sum of terms of one sign loses up to 2^-23 of its value by each 16 bf16 (32
// e4m3) of k. fp32 results therefore are sums, in registers, of tensor memory's sums over SUM_CHUNKS chunks of k.
// bf16 results are such sums (of more chunks: 2^-15) from LONG_CHUNKS (16384 bf16) on, where a single sum has lost
// 2^-13 and at 500000 bf16 of k 2.3e-3, more than half of their half unit.
constexpr int SUM_CHUNKS = 8, BF16_SUM_CHUNKS = 64, LONG_CHUNKS = 256;
constexpr int SMEM_MAX = 232448, STAGES_MAX = 20;
constexpr int DIRECT_CHUNKS = 4;          // most chunks of k per CTA whose operands the result warps bring

// A tile's parameters for the result warps.
struct Slot {
  int64_t y, residual, pre, part;  // element offsets of the CTA's first row and the tile's first column
  int rows, cols;                  // of the operand from there on
  int which, c0, c1;               // product; chunks of k
  int g, m, n;                     // group, first row and column
};

// VIA: a tile's residual and results pass through shared memory, by TMA.
template <int CG, int BN, bool VIA>
struct Shape {
  static constexpr int COLSW = BN / 4;            // columns of a result warp
  static constexpr int ACCS = BN == 256 ? 2 : 4;  // accumulators in tensor memory
  static constexpr int SLOTS = VIA ? 3 : 4;  // tiles whose parameters (and residual) are at hand
  static constexpr int TILE = VIA ? 128 * BN * 2 : 0;
  static constexpr int A_BYTES = 128 * ROW, B_BYTES = BN / CG * ROW, STAGE = A_BYTES + B_BYTES;
  // after the stages: the slots, each with {bias, w_scale}[BN] and x_scale[128]; partial sums; barriers
  static constexpr int SLOT = sizeof(Slot) + (2 * BN + 128) * 4;
  static constexpr int SUMS = EPI_WARPS * 32 * 4, BARS = 512;
  // a_rows: of A's box, fewer than 128 where m has fewer (the MMAs then read past them, into what follows:
  // rows of the sums that nobody reads)
  static constexpr int stage(int a_rows) { return a_rows * ROW + B_BYTES; }
  static constexpr int smem(int stages, int a_rows, bool turn) {
    return 1024 + stages * stage(a_rows) + (128 - a_rows) * ROW + SLOTS * (TILE + SLOT) + SUMS + BARS +
           (turn ? EPI_WARPS * TURN : 0);
  }
  static constexpr int stages(int a_rows, bool turn) {
    int n = a_rows < 128 ? STAGES_MAX : 8;
    while (smem(n, a_rows, turn) > SMEM_MAX) --n;
    return n;
  }
};

// n / d for 0 <= n < 2^31 as a multiplication: with s = ceil(log2 d) and m = ceil(2^(31 + s) / d), n m /
// 2^(31 + s) is above n / d by less than n / (d 2^31) < 1 / d.
struct Divisor {
  uint32_t mul;
  int shift;
  __device__ __forceinline__ int operator()(int n) const {
    return (int)((uint64_t)(uint32_t)n * mul >> shift);
  }
};
Divisor divisor(int64_t d) {
  int s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), 31 + s};
}

// One product's part of a launch.
struct Problem {
  Epilogue e;
  float* part;  // partial sums [splits][groups][m][ldp] instead of results, or null
  int64_t ldp;
  int groups, m, n, tiles_m, tiles_n, tiles, units, splits, chunks, chunks_per_split;
  int parts;             // SPLIT: CTAs of a cluster (and splits is 1)
  const uint8_t *a_rows, *b_rows;            // DIRECT: the operands, and their strides and k in bytes
  int64_t a_group, a_ld, b_group, b_ld, k_bytes;
  Divisor by_split, by_group, by_panel, by_rest;  // splits, tiles, 8 tiles_n, rows of the last panel
  int a_bytes;               // of A's box per CTA and stage
  int az, bz;                // 0: one matrix for every group
  int a_mn, b_mn;            // rows run along m (n) instead of k
  int a_blocked, b_blocked;  // a 4-D map brings the 64-wide boxes of a stage together
  int rz;                    // VIA: 0: one residual for every group
  int y_align, res_align, pre_align;  // 32, 16, or 0: bytes that divide every row's start
};
template <int NP>
struct GemmParams {
  CUtensorMap a[NP], b[NP];
  CUtensorMap residual, y;  // VIA: boxes of 32 columns by 128 and 32 rows
  Problem p[NP];
  PartSums sums;
  int units, stages, stage_bytes, a_rows;  // a_rows: of A in a stage
  int sum_chunks;                          // of k per sum in tensor memory, where results are sums of such
  int* err;
};

// Bounded wait of a warp for a barrier's phase, as tc::mbar_wait, that leaves the issue slots to the result
// warps: a try suspends the thread for up to 20 us.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* code,
                                     int what) {
  const auto attempt = [&] {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(20000u)
        : "memory");
    return ok != 0;
  };
  bool ok = attempt();
  if (!ok) {
    const unsigned long long t0 = tc::globaltimer();
    while (!(ok = attempt()) && !*abort_flag)
      if (tc::globaltimer() - t0 > tc::WAIT_NS) {
        *abort_flag = 1;
        *code = what;
      }
  }
  return __all_sync(0xffffffffu, ok);  // (its lanes leave the same way: they go on to warp-wide operations)
}

template <int CG>
__device__ __forceinline__ void load3(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y,
                                      int z) {
  if constexpr (CG == 2) tc::tma_load_3d_cg2(dst, m, bar, x, y, z);
  else tc::tma_load_3d(dst, m, bar, x, y, z);
}
template <int CG>
__device__ __forceinline__ void load4(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y,
                                      int z, int w) {
  if constexpr (CG == 2)
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"((uint64_t)m), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
  else
    tc::tma_load_4d(dst, m, bar, x, y, z, w);
}
// D (+)= A B over one step of 32 bytes of k
template <int TYPE, int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  if constexpr (TYPE == LIPZ_BF16) {
    if constexpr (CG == 2) tc::tc_mma_cg2(d, a, b, idesc, acc);
    else tc::tc_mma(d, a, b, idesc, acc);
  } else if constexpr (CG == 2) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
  } else {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
  }
}
// fp32 accumulators; bf16 (format 1) or e4m3 (format 0) operands
template <int TYPE>
__device__ __forceinline__ uint32_t idesc(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | (TYPE == LIPZ_BF16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)a_mn << 15) |
         ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (CG == 2) tc::tc_commit_cg2(bar, 3);
  else tc::tc_commit(bar);
}
__device__ __forceinline__ void ld_v8(const void* p, uint32_t* r) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                 "=r"(r[7])
               : "l"(p)
               : "memory");
}

// 16 elements of this lane's row (two bf16 or one fp32 per word), from a column of a warp's 32 rows on: 32-
// or 16-byte accesses where the rows' starts allow, else turned in shared memory so that the lanes run along
// a row. rows, cols: what there is of the 32 and the 16.
template <typename T>
constexpr int WORDS = sizeof(T) * 4;
template <typename T>
__device__ __forceinline__ float element(const uint32_t* w, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
  return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}
template <typename T>
__device__ __forceinline__ void load_row(const T* base, int64_t ld, int rows, int cols, int align,
                                         float* turn, uint32_t* w) {
  const int lane = threadIdx.x & 31;
  constexpr int W = WORDS<T>;
  if (align && cols >= 16) {
    if (lane < rows) {
      const char* p = reinterpret_cast<const char*>(base + lane * ld);
      if (align == 32) {
#pragma unroll
        for (int i = 0; i < W; i += 8) ld_v8(p + 4 * i, w + i);
      } else {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
          const uint4 r = *reinterpret_cast<const uint4*>(p + 4 * i);
          w[i] = r.x, w[i + 1] = r.y, w[i + 2] = r.z, w[i + 3] = r.w;
        }
      }
    }
    return;
  }
  const int col = lane & 15;
  __syncwarp();
#pragma unroll 8
  for (int r = lane >> 4; r < 32; r += 2)
    turn[r * 17 + col] = r < rows && col < cols ? to_f<T>(base[r * ld + col]) : 0.f;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(turn[lane * 17 + i]);
    else w[i] = tc::pack_bf16(turn[lane * 17 + 2 * i], turn[lane * 17 + 2 * i + 1]);
  }
}
template <typename T>
__device__ __forceinline__ void store_row(T* base, int64_t ld, int rows, int cols, int align,
                                          float* turn, const float* v) {
  const int lane = threadIdx.x & 31;
  constexpr int W = WORDS<T>;
  if (align && cols >= 16) {
    if (lane >= rows) return;
    uint32_t w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
      else w[i] = tc::pack_bf16(v[2 * i], v[2 * i + 1]);
    }
    char* p = reinterpret_cast<char*>(base + lane * ld);
    if (align == 32) {
#pragma unroll
      for (int i = 0; i < W; i += 8)
        tc::st_global_v8(p + 4 * i, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]),
                         make_uint4(w[i + 4], w[i + 5], w[i + 6], w[i + 7]));
    } else {
#pragma unroll
      for (int i = 0; i < W; i += 4)
        *reinterpret_cast<uint4*>(p + 4 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
    return;
  }
  const int col = lane & 15;
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 16; ++e) turn[lane * 17 + e] = v[e];
  __syncwarp();
#pragma unroll 8
  for (int r = lane >> 4; r < 32; r += 2)
    if (r < rows && col < cols) base[r * ld + col] = from_f<T>(turn[r * 17 + col]);
}

__device__ __forceinline__ int64_t ceil_div_d(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A unit's place: which part of k of which tile; groups outermost, then panels of 8 tile rows, along which
// neighbouring CTAs share operands in L2.
struct Place {
  int g, mt, nt, split;
};
__device__ __forceinline__ Place place(const Problem& p, int unit) {
  const int t = p.by_split(unit), g = p.by_group(t), r = t - g * p.tiles;
  const int panel = p.by_panel(r), first = panel * 8, q = r - panel * 8 * p.tiles_n;
  const bool whole = first + 8 <= p.tiles_m;
  const int nt = whole ? q >> 3 : p.by_rest(q);
  return {g, first + q - nt * (whole ? 8 : p.tiles_m - first), nt, unit - t * p.splits};
}

// T: float where results (of either type) are sums of sums over sum_chunks, else bf16. FORWARD: K-major operands
// and the forward's epilogue, one product; else up to two plain products.
// VIA: the residual comes and the results leave by TMA, through shared memory. With row-per-lane accesses,
// whose 64-byte pieces reach memory one by one, results cost 12 us and a residual 25 more at 144 x 512 x 256
// -> 768 (tanh with residual 88 us in all; by TMA 62).
// SPLIT: a cluster of CTAs shares a tile, each with a part of k; their sums are added over the cluster's
// shared memory, each CTA finishing a part of the columns. One tile per cluster.
// DIRECT: the result warps bring the operands first, from rows that TMA does not take.
template <int TYPE, int CG, int BN, bool FORWARD, typename T, bool VIA, bool SPLIT, bool DIRECT>
__global__ void __launch_bounds__(THREADS, 1)
    k_gemm_op(const __grid_constant__ GemmParams<FORWARD ? 1 : 2> prm) {
  using S = Shape<CG, BN, VIA>;
  constexpr bool SUMS = sizeof(T) == 4;
  static_assert(!VIA || (FORWARD && !SUMS && S::COLSW == 32), "boxes of 32 bf16 columns");
  static_assert(!SPLIT || (FORWARD && CG == 1 && !VIA && 128 * (BN + 1) * 4 <= 5 * S::B_BYTES),
                "sums of a tile");
  constexpr int BM = 128 * CG, COLSW = S::COLSW, ACCS = S::ACCS, SLOTS = S::SLOTS;
  constexpr int CW = COLSW < 32 ? COLSW : 32;       // a result warp's columns at a time
  constexpr int KE = TYPE == LIPZ_BF16 ? 64 : 128;  // k of a stage
  extern __shared__ uint8_t smem_raw[];
  const int stages = prm.stages, stage_bytes = FORWARD ? prm.stage_bytes : S::STAGE;
  const int a_stage = FORWARD ? prm.a_rows * ROW : S::A_BYTES;
  const uint32_t raw = tc::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  // [SLOTS][BN / 32][128 rows][64 bytes]
  uint8_t* tiles = smem_raw + (base - raw) + stages * stage_bytes + (S::A_BYTES - a_stage);
  uint8_t* slots = tiles + SLOTS * S::TILE;
  float* s_sum = reinterpret_cast<float*>(slots + SLOTS * S::SLOT);
  uint64_t* bars = reinterpret_cast<uint64_t*>(slots + SLOTS * S::SLOT + S::SUMS);
  float* s_turn = reinterpret_cast<float*>(slots + SLOTS * S::SLOT + S::SUMS + S::BARS);
  const uint32_t bFull = tc::smem_u32(bars), bEmpty = bFull + 8 * STAGES_MAX;
  const uint32_t bAcc = bEmpty + 8 * STAGES_MAX, bFree = bAcc + 8 * ACCS;
  const uint32_t bSlot = bFree + 8 * ACCS, bRead = bSlot + 8 * SLOTS;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bars + 60);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 61);
  int* code = reinterpret_cast<int*>(bars + 62);
  static_assert(2 * STAGES_MAX + 2 * ACCS + 2 * SLOTS <= 60, "barriers");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_ctarank() : 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      tc::mbar_init(bFull + 8 * s, DIRECT ? EPI_WARPS : 2);  // who brings: all, or A's and B's issuers
      tc::mbar_init(bEmpty + 8 * s, 1);
    }
    for (int r = 0; r < ACCS; ++r) {
      tc::mbar_init(bAcc + 8 * r, 1);
      tc::mbar_init(bFree + 8 * r, EPI_WARPS * CG);
    }
    for (int r = 0; r < SLOTS; ++r) {
      tc::mbar_init(bSlot + 8 * r, 1);
      tc::mbar_init(bRead + 8 * r, EPI_WARPS);
    }
    *abort_flag = 0;
    *code = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       tc::smem_u32((const void*)tmem_slot)),
                   "n"(ACCS * BN));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       tc::smem_u32((const void*)tmem_slot)),
                   "n"(ACCS * BN));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
  }
  tc::tc_fence_before();
  if constexpr (CG == 2) tc::cluster_sync_all();
  else __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t lFull = CG == 2 ? tc::mapa_shared(bFull, 0) : bFull;
  const uint32_t lFree = CG == 2 ? tc::mapa_shared(bFree, 0) : bFree;
  const int first = CG == 2 || SPLIT ? (int)tc::cluster_id_x() : (int)blockIdx.x;
  const int step = CG == 2 || SPLIT ? (int)tc::nclusters_x() : (int)gridDim.x;
  float* s_part = reinterpret_cast<float*>(smem_raw + (base - raw));  // SPLIT: [128][BN + 1], over the stages
  // The place of the warp's i-th unit: its lanes work out 32 units' places at a time.
  Place ahead{};
  auto unit_place = [&](int i) {
    if ((i & 31) == 0) {
      int unit = min(first + (i + lane) * step, prm.units - 1);
      const int which = !FORWARD && unit >= prm.p[0].units;
      if (which) unit -= prm.p[0].units;
      ahead = place(prm.p[which], unit);
      ahead.g |= which << 30;
    }
    const int from = i & 31;
    Place r{__shfl_sync(0xffffffffu, ahead.g, from), __shfl_sync(0xffffffffu, ahead.mt, from),
            __shfl_sync(0xffffffffu, ahead.nt, from), __shfl_sync(0xffffffffu, ahead.split, from)};
    if (SPLIT) r.split = (int)tc::cluster_ctarank();
    return r;
  };
  auto problem_of = [&](const Place& pl) -> const Problem& {
    return prm.p[FORWARD ? 0 : pl.g >> 30];
  };
  const int my_units = first < prm.units ? (prm.units - first + step - 1) / step : 0;
  auto chunk_range = [&](const Problem& p, int split, int& c0, int& c1) {
    c0 = split * p.chunks_per_split;
    c1 = min(p.chunks, c0 + p.chunks_per_split);
  };
  pdl_wait();

  if (DIRECT && warp < 2) {
  } else if (warp < 2) {
    // ============ TMA: warp 0 loads A, warp 1 loads B (both CTAs of a pair) ============
    const bool elected = tc::elect_one(), is_a = warp == 0;
    const int rows = is_a ? 128 : BN / CG;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int i = 0; i < my_units && ok; ++i) {
      const Place pl = unit_place(i);
      const Problem& p = problem_of(pl);
      const int which = FORWARD ? 0 : pl.g >> 30;
      const CUtensorMap* map = is_a ? &prm.a[which] : &prm.b[which];
      const bool mn = !FORWARD && (is_a ? p.a_mn : p.b_mn), blocked = is_a ? p.a_blocked : p.b_blocked;
      const uint32_t bytes = is_a && !mn ? (uint32_t)p.a_bytes : (uint32_t)(rows * ROW);
      const int at = is_a ? pl.mt * BM + (int)rank * 128 : pl.nt * BN + (int)rank * (BN / CG);
      const int z = (pl.g & 0x3FFFFFFF) * (is_a ? p.az : p.bz);
      int c0, c1;
      chunk_range(p, pl.split, c0, c1);
      for (int kc = c0; kc < c1; ++kc) {
        if (!wait(bEmpty + 8 * stage, phase ^ 1u, abort_flag, code, 1)) {
          ok = false;
          break;
        }
        const uint32_t dst = base + stage * stage_bytes + (is_a ? 0 : a_stage);
        const uint32_t full = lFull + 8 * stage;
        if (elected) {
          // the leader expects both CTAs' bytes; the peer's may land first
          if (rank == 0) tc::mbar_expect_tx(bFull + 8 * stage, CG * bytes);
          if (!mn) {
            load3<CG>(dst, map, full, kc * KE, at, z);
          } else if (blocked) {
            load4<CG>(dst, map, full, 0, kc * KE, at >> 6, z);
          } else {
            for (int h = 0; h < rows / 64; ++h)
              load3<CG>(dst + h * MN_BOX, map, full, at + 64 * h, kc * KE, z);
          }
        }
        if (++stage == stages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    if (!ok) {  // loads in flight land before the CTA leaves
      const unsigned long long t0 = tc::globaltimer();
      while (tc::globaltimer() - t0 < 200000ull) {
      }
    }
  } else if (warp == 2) {
    // ============ MMAs (rank 0) ============
    if (rank == 0) {
      const bool elected = tc::elect_one();
      int stage = 0, sums = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = 0; i < my_units && ok; ++i) {
        const Place pl = unit_place(i);
        const Problem& p = problem_of(pl);
        const int a_mn = FORWARD ? 0 : p.a_mn, b_mn = FORWARD ? 0 : p.b_mn;
        const uint32_t id = idesc<TYPE>(BM, BN, a_mn, b_mn);
        // a step further along k, in 16-byte units: 32 bytes of a row, or 16 rows of 128 bytes
        const uint32_t ia = a_mn ? 128 : 2, ib = b_mn ? 128 : 2;
        int c0, c1;
        chunk_range(p, pl.split, c0, c1);
        for (int kc = c0; kc < c1 && ok;) {
          const int end = SUMS ? min(c1, kc + prm.sum_chunks) : c1, r = sums % ACCS;
          if (sums >= ACCS &&
              !wait(bFree + 8 * r, (uint32_t)(sums / ACCS - 1) & 1, abort_flag, code, 2)) {
            ok = false;
            break;
          }
          tc::tc_fence_after();
          const uint32_t d = tmem + (uint32_t)(r * BN);
          for (uint32_t acc = 0; kc < end; ++kc) {
            if (!wait(bFull + 8 * stage, phase, abort_flag, code, 3)) {
              ok = false;
              break;
            }
            tc::tc_fence_after();
            const uint32_t sA = base + stage * stage_bytes, sB = sA + a_stage;
            const uint64_t dA = a_mn ? tc::sw128_mn_desc(sA, MN_BOX) : tc::sw128_desc(sA);
            const uint64_t dB = b_mn ? tc::sw128_mn_desc(sB, MN_BOX) : tc::sw128_desc(sB);
            if (elected) {
#pragma unroll
              for (int j = 0; j < 4; ++j) mma<TYPE, CG>(d, dA + j * ia, dB + j * ib, id, acc | (uint32_t)j);
              commit<CG>(bEmpty + 8 * stage);
            }
            acc = 1;
            if (++stage == stages) {
              stage = 0;
              phase ^= 1u;
            }
          }
          if (!ok) break;
          if (elected) commit<CG>(bAcc + 8 * r);
          ++sums;
        }
      }
    }
  } else if (warp == 3) {
    // ============ the tiles' parameters, as far ahead as there are slots ============
    bool ok = true;
    for (int i = 0; i < my_units && ok; ++i) {
      const Place pl = unit_place(i);
      const Problem& p = problem_of(pl);
      const Epilogue& e = p.e;
      const int64_t g = pl.g & 0x3FFFFFFF;
      const int row0 = pl.mt * BM + (int)rank * 128, n0 = pl.nt * BN;
      int c0, c1;
      chunk_range(p, pl.split, c0, c1);
      float bias[BN / 32], ws[BN / 32], xs[4];
      if (FORWARD && !SPLIT) {
#pragma unroll
        for (int j = 0; j < BN / 32; ++j) {
          const int n = n0 + j * 32 + lane;
          bias[j] = e.bias.data && n < p.n ? __ldg(e.bias.data + g * e.bias.group + n) : 0.f;
          if (TYPE == LIPZ_E4M3) ws[j] = n < p.n ? __ldg(e.w_scale.data + g * e.w_scale.group + n) : 1.f;
        }
        if (TYPE == LIPZ_E4M3) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int m = row0 + j * 32 + lane;
            xs[j] = m < p.m ? __ldg(e.x_scale.data + g * e.x_scale.group + m) : 1.f;
          }
        }
      }
      const int r = i % SLOTS;
      if (i >= SLOTS && !wait(bRead + 8 * r, (uint32_t)(i / SLOTS - 1) & 1, abort_flag, code, 5)) {
        ok = false;
        break;
      }
      uint8_t* slot = slots + r * S::SLOT;
      if (lane == 0)
        *reinterpret_cast<Slot*>(slot) =
            Slot{g * e.y.group + (int64_t)row0 * e.y.row + n0,
                 g * e.residual.group + (int64_t)row0 * e.residual.row + n0,
                 g * e.pre.group + (int64_t)row0 * e.pre.row + n0,
                 (((int64_t)pl.split * p.groups + g) * p.m + row0) * p.ldp + n0, p.m - row0, p.n - n0,
                 FORWARD ? 0 : pl.g >> 30, c0, c1, (int)g, row0, n0};
      if (FORWARD && !SPLIT) {
        float* f = reinterpret_cast<float*>(slot + sizeof(Slot));
#pragma unroll
        for (int j = 0; j < BN / 32; ++j) {
          f[j * 32 + lane] = bias[j];
          if (TYPE == LIPZ_E4M3) f[BN + j * 32 + lane] = ws[j];
        }
        if (TYPE == LIPZ_E4M3) {
#pragma unroll
          for (int j = 0; j < 4; ++j) f[2 * BN + j * 32 + lane] = xs[j];
        }
      }
      __syncwarp();
      if (VIA && e.residual.data) {
        if (lane == 0) {
          const uint32_t bar = bSlot + 8 * r, dst = tc::smem_u32(tiles + r * S::TILE);
          tc::mbar_expect_tx(bar, S::TILE);
#pragma unroll
          for (int j = 0; j < BN / 32; ++j)
            tc::tma_load_3d(dst + j * (S::TILE / (BN / 32)), &prm.residual, bar, n0 + j * 32, row0,
                            (int)g * p.rz);
        }
      } else if (lane == 0) {
        tc::mbar_arrive(bSlot + 8 * r);
      }
    }
    if (!ok) {  // loads in flight land before the CTA leaves
      const unsigned long long t0 = tc::globaltimer();
      while (tc::globaltimer() - t0 < 200000ull) {
      }
    }
  } else {
    // ============ results: a warp has 32 rows and a quarter of the tile's columns ============
    const int ew = warp - FIRST_EPI, q = warp & 3, col0 = (ew >> 2) * COLSW;
    float* turn = s_turn + ew * (TURN / 4);
    auto barrier = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory"); };
    if (!FORWARD && prm.sums.part) {
      // 32 columns of partial sums at a time, beside the first MMAs: every warp adds a 16th of the parts
      const PartSums& ps = prm.sums;
      const int64_t per = ceil_div_d(ps.cols, 32), blocks = per * ps.groups;
      for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t g = b / per, c = (b - g * per) * 32 + lane;
        float v = 0.f;
        if (c < ps.cols) {
          const float* src = ps.part + g * ps.parts * ps.cols + c;
#pragma unroll 8
          for (int i = ew; i < ps.parts; i += EPI_WARPS) v += src[i * ps.cols];
        }
        s_sum[ew * 32 + lane] = v;
        barrier();
        if (ew == 0 && c < ps.cols) {
          v = 0.f;
#pragma unroll
          for (int i = 0; i < EPI_WARPS; ++i) v += s_sum[i * 32 + lane];
          ps.out.data[g * ps.out.group + c] = v;
        }
        barrier();
      }
    }
    int sums = 0;
    bool ok = true;
    if constexpr (DIRECT) {
      static_assert(SPLIT, "one unit");
      const Problem& p = prm.p[0];
      const Place pl = unit_place(0);
      const int rows_a = min(prm.a_rows, p.m - pl.mt * BM);
      const int units = (rows_a + min(BN, p.n - pl.nt * BN)) * 8;
      const uint8_t* a = p.a_rows + pl.g * p.a_group + (int64_t)(pl.mt * BM) * p.a_ld;
      const uint8_t* b = p.b_rows + pl.g * p.b_group + (int64_t)(pl.nt * BN) * p.b_ld;
      int c0, c1;
      chunk_range(p, pl.split, c0, c1);
      for (int kc = c0; kc < c1 && ok; ++kc) {
        const int stage = (kc - c0) % stages;
        ok = wait(bEmpty + 8 * stage, (uint32_t)((kc - c0) / stages & 1) ^ 1u, abort_flag, code, 1);
        const uint32_t dst = base + stage * stage_bytes;
#pragma unroll 2
        for (int i = ew * 32 + lane; i < units; i += 32 * EPI_WARPS) {
          const int r = i >> 3, u = i & 7, rb = r - rows_a;
          const int64_t at = (int64_t)kc * ROW + u * 16;
          const uint4 v = bytes16(rb < 0 ? a + r * p.a_ld + at : b + rb * p.b_ld + at, p.k_bytes - at);
          const int row = rb < 0 ? r : rb;
          const uint32_t to = dst + (rb < 0 ? 0 : a_stage) + row * ROW + ((u ^ (row & 7)) << 4);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z),
                       "r"(v.w)
                       : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bFull + 8 * stage);
      }
    }
    auto wait_sum = [&]() {
      ok = wait(bAcc + 8 * (sums % ACCS), (uint32_t)(sums / ACCS) & 1, abort_flag, code, 4);
      tc::tc_fence_after();
      return tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(sums % ACCS * BN + col0);
    };
    auto free_sum = [&]() {
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) tc::mbar_arrive_remote(lFree + 8 * (sums % ACCS));
        else tc::mbar_arrive(bFree + 8 * (sums % ACCS));
      }
      ++sums;
    };
    for (int i = 0; i < my_units; ++i) {
      const int r = i % SLOTS;
      ok = wait(bSlot + 8 * r, (uint32_t)(i / SLOTS) & 1, abort_flag, code, 6);
      if (!ok) break;
      const uint8_t* slot = slots + r * S::SLOT;
      const Slot sl = *reinterpret_cast<const Slot*>(slot);
      const float* col = reinterpret_cast<const float*>(slot + sizeof(Slot)) + col0;
      const Problem& p = prm.p[FORWARD ? 0 : sl.which];
      const Epilogue& e = p.e;
      const int rows = sl.rows - q * 32;
      const float xs = TYPE == LIPZ_E4M3 && FORWARD && !SPLIT ? col[2 * BN - col0 + q * 32 + lane] : 1.f;
      // CW results of this lane's row, from column c of the warp's; v: the residual
      auto columns_left = [&](int c) { return sl.cols - (col0 + c); };
      constexpr int VW = CW / 16 * WORDS<T>;
      const bool has_res = FORWARD && !SPLIT && e.residual.data && rows > 0;
      // VIA: this lane's 64 bytes of the warp's 32 rows, 16-byte units in the 64-byte swizzle
      uint8_t* mine = tiles + r * S::TILE + (ew >> 2) * (S::TILE / (BN / 32)) + q * 2048 + lane * 64;
      const int swizzle = lane >> 1 & 3;
      const bool as_bf16 = SUMS && e.y.type == LIPZ_BF16;
      auto residual = [&](uint32_t (&v)[VW], int c) {
        if (VIA || !has_res) return;
        const int64_t at = sl.residual + (int64_t)(q * 32) * e.residual.row + col0 + c;
#pragma unroll
        for (int h = 0; h < CW; h += 16) {
          const int cols = columns_left(c + h);
          if (cols <= 0) continue;
          if (as_bf16)
            load_row<bf16>((const bf16*)e.residual.data + at + h, e.residual.row, rows, cols, p.res_align, turn,
                           v + h / 16 * WORDS<bf16>);
          else
            load_row<T>((const T*)e.residual.data + at + h, e.residual.row, rows, cols, p.res_align, turn,
                        v + h / 16 * WORDS<T>);
        }
      };
      auto results = [&](float (&u)[CW], const uint32_t (&v)[VW], int c) {
        if (rows <= 0 || columns_left(c) <= 0) return;
        if constexpr (SPLIT) {
          float* dst = s_part + (q * 32 + lane) * (BN + 1) + col0 + c;
#pragma unroll
          for (int j = 0; j < CW; ++j) dst[j] = u[j];
          return;
        }
        if (!FORWARD && p.part) {
          float* dst = p.part + sl.part + (int64_t)(q * 32) * p.ldp + col0 + c;
#pragma unroll
          for (int h = 0; h < CW; h += 16)
            if (columns_left(c + h) > 0)
              // (ldp is a multiple of 16: whole vectors)
              store_row<float>(dst + h, p.ldp, rows, 16, 32, turn, u + h);
          return;
        }
        if constexpr (FORWARD) {
#pragma unroll
          for (int i = 0; i < CW; i += 4) {
            const float4 b4 = *reinterpret_cast<const float4*>(col + c + i);
            uint64_t lo = pack2(u[i], u[i + 1]), hi = pack2(u[i + 2], u[i + 3]);
            if (TYPE == LIPZ_E4M3) {
              const float4 w4 = *reinterpret_cast<const float4*>(col + BN + c + i);
              lo = fma2(mul2(lo, both(xs)), pack2(w4.x, w4.y), pack2(b4.x, b4.y));
              hi = fma2(mul2(hi, both(xs)), pack2(w4.z, w4.w), pack2(b4.z, b4.w));
            } else {
              lo = add2(lo, pack2(b4.x, b4.y));
              hi = add2(hi, pack2(b4.z, b4.w));
            }
            const float2 l = unpack2(lo), h = unpack2(hi);
            u[i] = l.x, u[i + 1] = l.y, u[i + 2] = h.x, u[i + 3] = h.y;
          }
          if (e.pre.data) {
            bf16* dst = (bf16*)e.pre.data + sl.pre + (int64_t)(q * 32) * e.pre.row + col0 + c;
#pragma unroll
            for (int h = 0; h < CW; h += 16)
              if (columns_left(c + h) > 0)
                store_row<bf16>(dst + h, e.pre.row, rows, columns_left(c + h), p.pre_align, turn, u + h);
          }
          with_act(e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < CW; i += 2) act_pair<decltype(act)::value, SUMS>(u[i], u[i + 1], e.slope);
          });
          if (VIA && has_res) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint4 w = *reinterpret_cast<const uint4*>(mine + ((j ^ swizzle) << 4));
              const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int i = 0; i < 8; ++i) u[j * 8 + i] += element<T>(ww, i);
            }
          } else if (has_res && as_bf16) {
#pragma unroll
            for (int i = 0; i < CW; ++i) u[i] += element<bf16>(v + i / 16 * WORDS<bf16>, i % 16);
          } else if (has_res) {
#pragma unroll
            for (int i = 0; i < CW; ++i) u[i] += element<T>(v + i / 16 * WORDS<T>, i % 16);
          }
        }
        if constexpr (VIA) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<uint4*>(mine + ((j ^ swizzle) << 4)) =
                make_uint4(tc::pack_bf16(u[j * 8], u[j * 8 + 1]), tc::pack_bf16(u[j * 8 + 2], u[j * 8 + 3]),
                           tc::pack_bf16(u[j * 8 + 4], u[j * 8 + 5]),
                           tc::pack_bf16(u[j * 8 + 6], u[j * 8 + 7]));
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0)
            tc::tma_store_3d(&prm.y, tc::smem_u32(mine), sl.n + col0, sl.m + q * 32, sl.g);
          return;
        }
        const int64_t at = sl.y + (int64_t)(q * 32) * e.y.row + col0 + c;
#pragma unroll
        for (int h = 0; h < CW; h += 16) {
          const int cols = columns_left(c + h);
          if (cols <= 0) continue;
          if (as_bf16) store_row<bf16>((bf16*)e.y.data + at + h, e.y.row, rows, cols, p.y_align, turn, u + h);
          else store_row<T>((T*)e.y.data + at + h, e.y.row, rows, cols, p.y_align, turn, u + h);
        }
      };
      auto tmem_load = [&](uint32_t t, float (&u)[CW]) {
        uint32_t r[CW];
        if constexpr (CW == 32) LIPZ_TMEM_LD32(t, r);
        else LIPZ_TMEM_LD16(t, r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < CW; ++i) u[i] = __uint_as_float(r[i]);
      };
      uint32_t v[VW];
      if constexpr (SUMS) {
        static_assert(COLSW == CW, "the sums of a warp's columns stand in registers");
        float acc[CW];
#pragma unroll
        for (int i = 0; i < CW; ++i) acc[i] = 0.f;
        for (int kc = sl.c0; kc < sl.c1; kc += prm.sum_chunks) {
          const uint32_t t = wait_sum();
          if (!ok) break;
          float u[CW];
          tmem_load(t, u);
          free_sum();
#pragma unroll
          for (int i = 0; i < CW; ++i) acc[i] += u[i];
        }
        if (!ok) break;
        residual(v, 0);
        results(acc, v, 0);
      } else {
        residual(v, 0);
        const uint32_t t = wait_sum();
        if (!ok) break;
#pragma unroll 1
        for (int c = 0; c < COLSW; c += CW) {
          float u[CW];
          tmem_load(t + c, u);
          if (c + CW == COLSW) free_sum();
          uint32_t cur[VW];
#pragma unroll
          for (int i = 0; i < VW; ++i) cur[i] = v[i];
          if (c + CW < COLSW) residual(v, c + CW);
          results(u, cur, c);
        }
      }
      if (VIA) {
        // a slot is free again when the stores of the warp's tile before this one have read it
        if (lane == 0) {
          tc::bulk_commit();
          tc::bulk_wait_read<1>();
          if (i) tc::mbar_arrive(bRead + 8 * ((i - 1) % SLOTS));
        }
        __syncwarp();
        continue;
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bRead + 8 * r);
    }
    if (VIA && lane == 0) tc::bulk_wait_all();
  }
  if constexpr (SPLIT) {
    __syncwarp();
    tc::cluster_sync_all();  // every CTA's sums stand in its shared memory
    const Problem& p = prm.p[0];
    const Place pl = place(p, first);
    const int parts = p.parts, rows = min(128, p.m - pl.mt * 128), width = BN / parts;
    const int c0 = (int)tc::cluster_ctarank() * width;
    for (int i = threadIdx.x; i < rows * width; i += THREADS) {
      const int r = i / width, c = c0 + i - r * width, n = pl.nt * BN + c;
      if (n >= p.n) continue;
      const uint32_t at = tc::smem_u32(s_part + r * (BN + 1) + c);
      float u = 0.f;
      for (int j = 0; j < parts; ++j) {
        float v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::mapa_shared(at, j)) : "memory");
        u += v;
      }
      finish(p.e, pl.g, pl.mt * 128 + r, n, u);
    }
  }
  tc::tc_fence_before();
  __syncwarp();
  if constexpr (CG == 2 || SPLIT) tc::cluster_sync_all();  // (SPLIT: no CTA leaves while its sums are read)
  else __syncthreads();
  tc::tc_fence_after();
  if (warp == 2) {
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(ACCS * BN));
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(ACCS * BN));
  }
  if (threadIdx.x == 0 && *code && prm.err) *reinterpret_cast<volatile int*>(prm.err) = *code;
}

// Sum of the parts of k, in order. E columns per thread.
struct FinishParams {
  lipz_mat y;
  const float* part;
  int64_t ldp, split_stride, total;  // rows of all groups
  int splits, m, n;
};
struct FinishPair {
  FinishParams f[2];
};
template <int E>
__global__ void __launch_bounds__(256) k_finish(const __grid_constant__ FinishPair both_p) {
  const FinishParams& p = both_p.f[blockIdx.z];
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  if (r >= p.total) return;
  const int64_t g = r / p.m, o = g * p.y.group + (r - g * p.m) * p.y.row;
  for (int64_t c = ((int64_t)blockIdx.y * 32 + (threadIdx.x & 31)) * E; c < p.n;
       c += (int64_t)gridDim.y * 32 * E) {
    float u[E];
#pragma unroll
    for (int i = 0; i < E; ++i) u[i] = 0.f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
      const float* q = p.part + s * p.split_stride + r * p.ldp + c;
      if constexpr (E == 4) {
        const float4 v = *reinterpret_cast<const float4*>(q);
        u[0] += v.x, u[1] += v.y, u[2] += v.z, u[3] += v.w;
      } else {
        u[0] += *q;
      }
    }
    if (p.y.type == LIPZ_FP32) {
      float* y = (float*)p.y.data + o + c;
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = u[i];
    } else {
      bf16* y = (bf16*)p.y.data + o + c;
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = __float2bfloat16_rn(u[i]);
    }
  }
}

__global__ void __launch_bounds__(256) k_copy_rows(const __grid_constant__ CopyJobs jobs) {
  pdl_wait();
  copy_rows(jobs, blockIdx.x);
}

// Blocks of 8 rows by 32 columns' threads; columns past 65535 blocks are looped over.
dim3 rows_by_columns(int64_t rows, int64_t columns) {
  const int64_t y = ceil_div(columns, 32);
  return dim3((unsigned)ceil_div(rows, 8), (unsigned)(y < 65535 ? y : 65535));
}

// ---- host ----------------------------------------------------------------------------------------

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 f = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
            cudaSuccess || q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      fn = nullptr;
    }
    return (PFN_cuTensorMapEncodeTiled_v12000)fn;
  }();
  return f;
}

// rows, cols: an operand's matrix as it lies in memory
struct Extent {
  int64_t rows, cols;
};
Extent extent(const Operand& o, int64_t mn, int64_t k) {
  return o.k_major ? Extent{mn, k} : Extent{k, mn};
}

// Whether TMA takes the matrices as they lie: rows and groups on 16-byte boundaries, rows not overlapping.
bool tma_takes(const Operand& o, const Extent& x, int64_t groups, int eb) {
  if ((uintptr_t)o.data % 16) return false;
  if (x.rows > 1 && (o.ld * eb % 16 || o.ld < x.cols || o.ld * eb >= (int64_t)1 << 40)) return false;
  return groups == 1 || (o.group * eb % 16 == 0 && o.group * eb < (int64_t)1 << 40);
}

// An operand that the groups share is copied once (144 groups of 100 x 777 -> 501: 76 -> 38 us).
int64_t copied_groups(const Operand& o, int64_t groups) { return o.group ? groups : 1; }

// The map of results or a residual, {n, m, groups}, in boxes of 32 bf16 columns.
bool encode_tile(CUtensorMap* map, const lipz_mat& m, int64_t rows, int64_t cols, int64_t groups,
                 int box_rows) {
  const auto f = encoder();
  if (!f) return false;
  const cuuint64_t row = rows > 1 ? (cuuint64_t)m.row * 2 : (cuuint64_t)ceil_div(cols, 8) * 16;
  const cuuint64_t depth = groups > 1 && m.group ? (cuuint64_t)groups : 1;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, depth};
  const cuuint64_t strides[2] = {row, depth > 1 ? (cuuint64_t)m.group * 2 : row};
  const cuuint32_t box[3] = {32, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, m.data, dims, strides, box, es,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The map of an operand: {cols, rows, groups} in boxes of one 128-byte unit by box_rows rows; blocked:
// {64, rows, cols / 64, groups} in boxes of 64 x 64 x blocks.
bool encode(CUtensorMap* map, const Operand& o, const Extent& x, int64_t groups, int type, int box_rows,
            int blocks) {
  const auto f = encoder();
  if (!f) return false;
  const int eb = type_bytes(type);
  const cuuint64_t units = (cuuint64_t)ceil_div(x.cols * eb, 16) * 16;
  const cuuint64_t row = x.rows > 1 ? (cuuint64_t)o.ld * eb : units;
  const cuuint64_t depth = groups > 1 && o.group ? (cuuint64_t)groups : 1;
  const cuuint64_t group = depth > 1 ? (cuuint64_t)o.group * eb : row;
  const CUtensorMapDataType t =
      type == LIPZ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const cuuint32_t es[4] = {1, 1, 1, 1};
  CUresult r;
  if (blocks) {
    const cuuint64_t dims[4] = {64, (cuuint64_t)x.rows, (cuuint64_t)(x.cols / 64), depth};
    const cuuint64_t strides[3] = {row, 128, group};
    const cuuint32_t box[4] = {64, 64, (cuuint32_t)blocks, 1};
    r = f(map, t, 4, const_cast<void*>(o.data), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else {
    const cuuint64_t dims[3] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows, depth};
    const cuuint64_t strides[2] = {row, group};
    const cuuint32_t box[3] = {(cuuint32_t)(ROW / eb), (cuuint32_t)box_rows, 1};
    r = f(map, t, 3, const_cast<void*>(o.data), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  }
  return r == CUDA_SUCCESS;
}

uint64_t round256(int64_t v) { return (uint64_t)ceil_div(v, 256) * 256; }

template <int TYPE, int CG, int BN, bool FORWARD, typename T, bool VIA = false, bool SPLIT = false,
          bool DIRECT = false>
cudaError_t launch(const Products& q, const GemmPlan& plan, float* const* parts, const PartSums* sums,
                   cudaStream_t st) {
  using S = Shape<CG, BN, VIA>;
  GemmParams<FORWARD ? 1 : 2> k;
  memset(&k, 0, sizeof k);
  bool turn = false;
  for (int i = 0; i < q.n; ++i) {
    const Gemm& g = q.g[i];
    const GemmPlan::One& o = plan.p[i];
    Problem& p = k.p[i];
    const Extent xa = extent(g.a, g.m, g.k), xb = extent(g.b, g.n, g.k);
    p.a_mn = !g.a.k_major, p.b_mn = !g.b.k_major;
    p.a_blocked = p.a_mn && g.m % 64 == 0;
    p.b_blocked = p.b_mn && g.n % 64 == 0;
    const int arows = p.a_mn ? 64 : (int)(g.m >= 128 ? 128 : ceil_div(g.m, 8) * 8);
    const int brows = p.b_mn ? 64 : BN / CG;
    if (DIRECT) {
      const int eb = type_bytes(TYPE);
      p.a_rows = (const uint8_t*)g.a.data, p.b_rows = (const uint8_t*)g.b.data;
      p.a_group = g.a.group * eb, p.a_ld = g.a.ld * eb, p.b_group = g.b.group * eb, p.b_ld = g.b.ld * eb;
      p.k_bytes = g.k * eb;
    } else if (!encode(&k.a[i], g.a, xa, g.groups, TYPE, arows, p.a_blocked ? 2 : 0) ||
               !encode(&k.b[i], g.b, xb, g.groups, TYPE, brows, p.b_blocked ? BN / CG / 64 : 0))
      return cudaErrorInvalidValue;
    p.e = g.e;
    p.part = parts[i];
    p.ldp = o.ldp;
    p.groups = (int)g.groups, p.m = (int)g.m, p.n = (int)g.n;
    p.tiles_m = (int)o.tiles_m, p.tiles_n = (int)o.tiles_n;
    p.splits = SPLIT ? 1 : o.splits;
    p.parts = o.splits;
    p.tiles = (int)(o.tiles_m * o.tiles_n);
    p.units = (int)(p.tiles * g.groups * p.splits);
    p.by_split = divisor(p.splits), p.by_group = divisor(p.tiles);
    p.by_panel = divisor(8 * o.tiles_n), p.by_rest = divisor(o.tiles_m % 8 ? o.tiles_m % 8 : 8);
    p.chunks = (int)o.chunks, p.chunks_per_split = (int)o.chunks_per_split;
    p.a_bytes = arows * ROW;
    p.az = g.groups > 1 && g.a.group != 0, p.bz = g.groups > 1 && g.b.group != 0;
    auto align = [&](const lipz_mat& m) {
      const int a = !m.data || rows_aligned(m, g.groups, g.m, 32) ? 32
                    : rows_aligned(m, g.groups, g.m, 16)          ? 16
                                                                  : 0;
      turn = turn || (m.data && !p.part && (!a || g.n % 16) && (!VIA || m.data == g.e.pre.data));
      return a;
    };
    p.y_align = align(g.e.y), p.res_align = align(g.e.residual), p.pre_align = align(g.e.pre);
    k.units += p.units;
    if (VIA) {
      p.rz = g.groups > 1 && g.e.residual.group != 0;
      if (!encode_tile(&k.y, g.e.y, g.m, g.n, g.groups, 32) ||
          (g.e.residual.data && !encode_tile(&k.residual, g.e.residual, g.m, g.n, g.groups, 128)))
        return cudaErrorInvalidValue;
    }
  }
  if (sums) k.sums = *sums;
  k.err = timeout_word();
  k.sum_chunks = q.g[0].e.y.type == LIPZ_FP32 ? SUM_CHUNKS : BF16_SUM_CHUNKS;
  const Gemm& first = q.g[0];
  k.a_rows = FORWARD && CG == 1 && first.m < 128 ? (int)ceil_div(first.m, 8) * 8 : 128;
  k.stage_bytes = S::stage(k.a_rows);
  k.stages = S::stages(k.a_rows, turn);
  static std::atomic<uint64_t> done{0};
  auto kernel = k_gemm_op<TYPE, CG, BN, FORWARD, T, VIA, SPLIT, DIRECT>;
  cudaError_t e = allow_dynamic_smem(kernel, SMEM_MAX, done);
  if (e != cudaSuccess) return e;
  const int cluster = SPLIT ? k.p[0].parts : CG, slots = SPLIT ? k.units : sm_count() / CG;
  const int ctas = (k.units < slots ? k.units : slots) * cluster;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = S::smem(k.stages, k.a_rows, turn);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  const bool shared = st == nullptr || st == cudaStreamLegacy || st == cudaStreamPerThread;
  cfg.attrs = attr;
  cfg.numAttrs = shared ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, kernel, k);
}

// Whether TMA takes a forward's bf16 results and residual as they lie.
bool results_by_tma(const Gemm& g) {
  auto takes = [&](const lipz_mat& m) {
    return !m.data || tma_takes({m.data, m.group, m.row, true}, {g.m, g.n}, g.groups, 2);
  };
  return g.e.y.type == LIPZ_BF16 && g.a.k_major && g.b.k_major && takes(g.e.y) && takes(g.e.residual);
}

template <int TYPE, bool FORWARD>
cudaError_t launch_shape(const Products& q, const GemmPlan& p, float* const* parts, const PartSums* sums,
                         cudaStream_t st) {
  if constexpr (FORWARD) {
    if (p.direct)
      return p.sums
                 ? launch<TYPE, 1, 64, true, float, false, true, true>(q, p, parts, sums, st)
                 : launch<TYPE, 1, 64, true, bf16, false, true, true>(q, p, parts, sums, st);
    if (p.p[0].splits > 1)
      return p.sums
                 ? launch<TYPE, 1, 64, true, float, false, true>(q, p, parts, sums, st)
                 : launch<TYPE, 1, 64, true, bf16, false, true>(q, p, parts, sums, st);
  }
  if (p.sums) {
    if (p.cg == 2) return launch<TYPE, 2, 128, FORWARD, float>(q, p, parts, sums, st);
    if (p.bn == 128) return launch<TYPE, 1, 128, FORWARD, float>(q, p, parts, sums, st);
    return launch<TYPE, 1, 64, FORWARD, float>(q, p, parts, sums, st);
  }
  if (p.cg == 2 && p.bn == 256) return launch<TYPE, 2, 256, FORWARD, bf16>(q, p, parts, sums, st);
  if constexpr (FORWARD) {
    if (p.cg == 2 && results_by_tma(q.g[0]))
      return launch<TYPE, 2, 128, true, bf16, true>(q, p, parts, sums, st);
  }
  if (p.cg == 2) return launch<TYPE, 2, 128, FORWARD, bf16>(q, p, parts, sums, st);
  if (p.bn == 128) return launch<TYPE, 1, 128, FORWARD, bf16>(q, p, parts, sums, st);
  return launch<TYPE, 1, 64, FORWARD, bf16>(q, p, parts, sums, st);
}

}  // namespace

GemmPlan plan_products(const Products& q) {
  GemmPlan plan{};
  const Gemm& g0 = q.g[0];
  const int eb = type_bytes(g0.type);
  const bool fp32 = g0.e.y.type == LIPZ_FP32, res = g0.e.residual.data, heavy = g0.e.act >= LIPZ_ACT_TANH;
  // The shape and the number of parts of k that take the fewest clocks by a model of a unit's time: its MMA
  // steps (of 32 bytes of k) beside the epilogue of the unit before; parts of k cost a cluster's exchange,
  // or another launch and their way through L2. Clocks measured (1.9 GHz): MMA steps at 8192 x 4096 -> 8192
  // in bf16 (8 bits: 184 instead of 158), epilogues at 144 x 512 x 256 -> 768 without an activation, what
  // tanh adds, what a residual adds.
  struct Shape {
    int cg, bn;
    double step, epi, act, residual;
  };
  static const Shape shapes[] = {{2, 256, 158, 9000, 2500, 5500}, {2, 128, 88, 3900, 800, 2600},
                                 {1, 128, 108, 3900, 800, 2600}, {1, 64, 82, 2350, 250, 900}};
  const Shape via{2, 128, 100, 3500, 400, 1000};  // shape 1 with its results through shared memory
  const bool by_tma = results_by_tma(g0), forward = g0.a.k_major && g0.b.k_major;
  const int sms = sm_count();
  double best = -1;
  for (const Shape& shape : shapes) {
    if (fp32 && shape.bn > 128) continue;
    // a forward's parts of k are a cluster's CTAs, all clusters resident at once
    for (int s0 = 1; s0 <= (forward ? 8 : 64); s0 *= 2) {
      if (forward && s0 > 1 && shape.bn != 64) continue;
      const Shape& c = by_tma && s0 == 1 && shape.cg == 2 && shape.bn == 128 ? via : shape;
      const int64_t slots = sms / c.cg;
      GemmPlan t{};
      t.cg = c.cg, t.bn = c.bn, t.sums = fp32;
      double work = 0, top = 0, last = 0, extra = 0;
      bool fits = true, split = false;
      for (int i = 0; i < q.n; ++i) {
        const Gemm& g = q.g[i];
        GemmPlan::One& o = t.p[i];
        o.tiles_m = ceil_div(g.m, 128 * c.cg), o.tiles_n = ceil_div(g.n, c.bn);
        o.chunks = ceil_div(g.k * eb, ROW);
        const int64_t want = s0 < o.chunks ? s0 : o.chunks, tiles = o.tiles_m * o.tiles_n * g.groups;
        o.chunks_per_split = ceil_div(o.chunks, want);
        o.splits = (int)ceil_div(o.chunks, o.chunks_per_split);
        t.sums = t.sums || o.chunks_per_split > LONG_CHUNKS;
        fits = fits && tiles * o.splits <= INT32_MAX / 2 &&
               (o.splits == 1 || tiles * o.splits <= (forward ? 1 : 2) * slots) &&
               (!forward || o.splits == s0);
        const double mma = o.chunks_per_split * 4 * c.step * (eb == 1 ? 1.16 : 1);
        const double epi = c.epi + (heavy ? c.act : 0) + (res ? c.residual : 0);
        const double unit = mma > epi ? mma : epi;
        work += unit * tiles * o.splits;
        if (unit > top) top = unit;
        if (mma + epi > last) last = mma + epi;
        if (o.splits > 1 && !forward) extra += (double)g.groups * g.m * g.n * 4 * o.splits * 2 / 3000;
        split = split || o.splits > 1;
      }
      if (!fits || (s0 > 1 && !split) || (t.sums && c.bn > 128)) continue;
      double waves = work / (slots * top);
      waves = waves < 1 ? 0 : (double)(int64_t)(waves + 0.999) - 1;
      // (a cluster's CTA finishes 64 / s0 columns of up to 128 rows, an element per thread and turn)
      const double join = 4500 + 70.0 / s0 * (g0.m < 128 ? g0.m : 128);
      const double time = waves * top + last + extra + (!split ? 0 : forward ? join : 9500);
      if (best < 0 || time < best) best = time, plan = t;
    }
  }
  if (forward) {
    // Rows that TMA does not take: brought by the result warps where one wave of small tiles is all, so that
    // no copies have to be made first (37 x 1000 -> 500 over 8-bit operands: 12 us with the copies' launch,
    // 8 without). As many parts of k as there are CTAs for.
    const Extent xa = extent(g0.a, g0.m, g0.k), xb = extent(g0.b, g0.n, g0.k);
    GemmPlan t{};
    GemmPlan::One& o = t.p[0];
    o.tiles_m = ceil_div(g0.m, 128), o.tiles_n = ceil_div(g0.n, 64), o.chunks = ceil_div(g0.k * eb, ROW);
    const int64_t tiles = o.tiles_m * o.tiles_n * g0.groups;
    if ((!tma_takes(g0.a, xa, g0.groups, eb) || !tma_takes(g0.b, xb, g0.groups, eb)) && tiles <= sms) {
      t.direct = true, t.sums = fp32, t.cg = 1, t.bn = 64;
      for (int s0 = 8; s0 >= 1; s0 /= 2) {
        o.chunks_per_split = ceil_div(o.chunks, s0 < o.chunks ? s0 : o.chunks);
        o.splits = (int)ceil_div(o.chunks, o.chunks_per_split);
        if (o.splits == s0 && tiles * s0 <= sms) break;
      }
      if (o.chunks_per_split <= DIRECT_CHUNKS) plan = t;
    }
  }
  plan_space(q, &plan);
  return plan;
}

void plan_space(const Products& q, GemmPlan* plan) {
  const int eb = type_bytes(q.g[0].type), unit = 16 / eb;
  plan->bytes = 0;
  for (int i = 0; i < q.n; ++i) {
    const Gemm& g = q.g[i];
    GemmPlan::One& o = plan->p[i];
    const Extent xa = extent(g.a, g.m, g.k), xb = extent(g.b, g.n, g.k);
    o.copy_a = !plan->direct && !tma_takes(g.a, xa, g.groups, eb);
    o.copy_b = !plan->direct && !tma_takes(g.b, xb, g.groups, eb);
    o.lda = ceil_div(xa.cols, unit) * unit;
    o.ldb = ceil_div(xb.cols, unit) * unit;
    o.a_bytes = o.copy_a ? round256(copied_groups(g.a, g.groups) * xa.rows * o.lda * eb) : 0;
    o.b_bytes = o.copy_b ? round256(copied_groups(g.b, g.groups) * xb.rows * o.ldb * eb) : 0;
    o.ldp = ceil_div(g.n, 16) * 16;
    const bool through_memory = o.splits > 1 && !(g.a.k_major && g.b.k_major);
    o.part_bytes = through_memory ? round256((int64_t)o.splits * g.groups * g.m * o.ldp * 4) : 0;
    plan->bytes += o.a_bytes + o.b_bytes + o.part_bytes;
  }
}

int plan_copies(const GemmPlan& plan, Products* q, void* workspace, RowCopy* copies) {
  char* w = (char*)workspace;
  int n = 0;
  for (int i = 0; i < q->n; ++i) {
    Gemm& g = q->g[i];
    const GemmPlan::One& o = plan.p[i];
    const int eb = type_bytes(g.type);
    auto add = [&](Operand& t, const Extent& x, int64_t ld, uint64_t bytes) {
      const int64_t groups = copied_groups(t, g.groups);
      copies[n++] = {(const uint8_t*)t.data, w, t.group * eb, t.ld * eb, x.rows, groups * x.rows, x.cols * eb,
                     ld * eb / 16};
      t.data = w, t.ld = ld, t.group = groups > 1 ? x.rows * ld : 0;
      w += bytes;
    };
    if (o.copy_a) add(g.a, extent(g.a, g.m, g.k), o.lda, o.a_bytes);
    if (o.copy_b) add(g.b, extent(g.b, g.n, g.k), o.ldb, o.b_bytes);
  }
  return n;
}

CopyJobs copy_jobs(const RowCopy* c, int n) {
  CopyJobs jobs{};
  jobs.n = n;
  for (int i = 0; i < n; ++i) {
    jobs.c[i] = c[i];
    jobs.blocks += ceil_div(c[i].total, COPY_ROWS);
  }
  return jobs;
}

cudaError_t run_copies(const CopyJobs& jobs, cudaStream_t st) {
  if (jobs.blocks == 0) return cudaSuccess;
  return launch_pdl(k_copy_rows, dim3((unsigned)jobs.blocks), dim3(256), 0, st, jobs);
}

cudaError_t run_products(const GemmPlan& plan, const Products& q, void* workspace, const PartSums* sums,
                         cudaStream_t st) {
  char* w = (char*)workspace;
  float* parts[2] = {nullptr, nullptr};
  for (int i = 0; i < q.n; ++i) w += plan.p[i].a_bytes + plan.p[i].b_bytes;
  for (int i = 0; i < q.n; ++i)
    if (plan.p[i].part_bytes) {
      parts[i] = (float*)w;
      w += plan.p[i].part_bytes;
    }
  const Gemm& g0 = q.g[0];
  cudaError_t e;
  if (g0.type == LIPZ_E4M3) e = launch_shape<LIPZ_E4M3, true>(q, plan, parts, sums, st);
  else if (g0.a.k_major && g0.b.k_major) e = launch_shape<LIPZ_BF16, true>(q, plan, parts, sums, st);
  else e = launch_shape<LIPZ_BF16, false>(q, plan, parts, sums, st);
  if (e != cudaSuccess || (!parts[0] && !parts[1])) return e;
  FinishPair f{};
  int n = 0;
  bool vec = true;
  int64_t rows = 0, cols = 0;
  for (int i = 0; i < q.n; ++i) {
    if (!parts[i]) continue;
    const Gemm& g = q.g[i];
    const int64_t ldp = plan.p[i].ldp;
    f.f[n++] = {g.e.y, parts[i], ldp, g.groups * g.m * ldp, g.groups * g.m, plan.p[i].splits, (int)g.m,
                (int)g.n};
    vec = vec && g.n % 4 == 0;
    rows = rows > g.groups * g.m ? rows : g.groups * g.m;
    cols = cols > g.n ? cols : g.n;
  }
  dim3 grid = rows_by_columns(rows, vec ? cols / 4 : cols);
  grid.z = n;
  return vec ? launch_pdl(k_finish<4>, grid, dim3(256), 0, st, f)
             : launch_pdl(k_finish<1>, grid, dim3(256), 0, st, f);
}

}  // namespace ops
}  // namespace lipz
