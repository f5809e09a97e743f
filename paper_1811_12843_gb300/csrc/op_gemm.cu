// Tensor-core product of the residual-block operators (tcgen05, sm_103a).
//
// A tile of C is BM x BN: 128 rows on one CTA, or 256 on a pair of CTAs whose MMAs take A's rows from both
// and half of B's rows from each (so that a byte of B that is brought from L2 serves 256 rows). Persistent
// CTAs walk over tiles (and parts of k); two warps issue the TMA loads of A and of B into a ring of
// 128-byte-swizzled stages, one issues the MMAs into one of two accumulators in tensor memory, and eight
// turn the other accumulator into results.
// Bound: the tensor cores for large sizes, the epilogue for k of a few hundred, HBM for few rows.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>
#include <type_traits>

#include "op_gemm.h"
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace lipz {
namespace ops {

namespace {

constexpr int ROW = 128;                  // bytes of a swizzled row: 64 bf16 or 128 e4m3 of k
constexpr int EPI_WARPS = 8, FIRST_EPI = 4, THREADS = 32 * (FIRST_EPI + EPI_WARPS);
constexpr int TURN = 32 * 17 * 4;         // a warp's block for turning rows into columns
constexpr int MN_BOX = 64 * ROW;          // 64 k by 64 m (or n) of an operand whose rows run along m (n)
constexpr int SUM_CHUNKS = 8;             // chunks of k whose sum stands in tensor memory, for fp32 results
constexpr int SMEM_MAX = 232448;

template <int CG, int BN>
struct Shape {
  static constexpr int A_BYTES = 128 * ROW, B_BYTES = BN / CG * ROW, STAGE = A_BYTES + B_BYTES;
  static constexpr int EXTRA = 1024 + EPI_WARPS * TURN + 2 * BN * 8 + 256;
  static constexpr int STAGES = (SMEM_MAX - EXTRA) / STAGE < 8 ? (SMEM_MAX - EXTRA) / STAGE : 8;
  static constexpr int SMEM = EXTRA + STAGES * STAGE;
};

struct GemmParams {
  Epilogue e;
  float* part;  // partial sums [splits][groups][m][ldp] instead of results, or null
  int* err;
  int64_t ldp;
  int groups, m, n, tiles_m, tiles_n, units, splits, chunks, chunks_per_split;
  int a_bytes;           // of A's box per CTA and stage
  int az, bz;            // 0: one matrix for every group
  int a_blocked, b_blocked;  // a 4-D map brings the 64-wide boxes of a stage together
  int y_align, res_align, pre_align;  // 32, 16, or 0: bytes that divide every row's start
};

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
__host__ __device__ constexpr uint32_t idesc(int m, int n, bool a_mn, bool b_mn) {
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

// 32 elements of this lane's row, from column c of a warp's 32 rows: 32- or 16-byte accesses where the
// rows' starts allow, else turned in shared memory so that the lanes run along a row. (rows, cols: what
// there is of the 32.) Words: two bf16, or one fp32.
template <typename T>
__device__ __forceinline__ void load_row(const T* base, int64_t ld, int rows, int cols, int align,
                                         float* turn, float (&v)[32]) {
  const int lane = threadIdx.x & 31;
  constexpr int W = sizeof(T) * 8;  // words of 32 elements
  if (align && cols >= 32) {
    uint32_t w[W];
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
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = 0;
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      if constexpr (sizeof(T) == 4) v[e] = __uint_as_float(w[e]);
      else v[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = h * 16 + (lane & 15);
    __syncwarp();
#pragma unroll 8
    for (int r = lane >> 4; r < 32; r += 2)
      turn[r * 17 + (lane & 15)] = r < rows && col < cols ? to_f<T>(base[r * ld + col]) : 0.f;
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 16; ++e) v[h * 16 + e] = turn[lane * 17 + e];
  }
}
template <typename T>
__device__ __forceinline__ void store_row(T* base, int64_t ld, int rows, int cols, int align,
                                          float* turn, const float (&v)[32]) {
  const int lane = threadIdx.x & 31;
  constexpr int W = sizeof(T) * 8;
  if (align && cols >= 32) {
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
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = h * 16 + (lane & 15);
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 16; ++e) turn[lane * 17 + e] = v[h * 16 + e];
    __syncwarp();
#pragma unroll 8
    for (int r = lane >> 4; r < 32; r += 2)
      if (r < rows && col < cols) base[r * ld + col] = from_f<T>(turn[r * 17 + (lane & 15)]);
  }
}

// A tile's place: groups outermost, then panels of 8 tile rows, along which neighbouring CTAs share
// operands in L2.
struct Place {
  int g, mt, nt;
};
__device__ __forceinline__ Place place(int t, int tiles_m, int tiles_n) {
  const int per = tiles_m * tiles_n, g = t / per, r = t - g * per;
  const int panel = r / (8 * tiles_n), first = panel * 8, w = min(8, tiles_m - first);
  const int q = r - panel * 8 * tiles_n;
  return {g, first + q % w, q / w};
}

// T: the results' type; fp32 results (SUMS) are sums, in fp32 registers, of sums over SUM_CHUNKS chunks,
// because the tensor cores' additions truncate. FORWARD: K-major operands and the forward's epilogue, else
// a plain product.
template <int TYPE, int CG, int BN, bool AMN, bool BMN, typename T>
__global__ void __launch_bounds__(THREADS, 1)
    k_gemm_op(const __grid_constant__ CUtensorMap mA, const __grid_constant__ CUtensorMap mB,
              const __grid_constant__ GemmParams p) {
  using S = Shape<CG, BN>;
  constexpr int STAGES = S::STAGES, BM = 128 * CG, HALF = BN / 2;
  constexpr bool SUMS = sizeof(T) == 4, FORWARD = !AMN && !BMN;
  constexpr int KE = TYPE == LIPZ_BF16 ? 64 : 128;  // k of a stage
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* after = smem_raw + (base - raw) + STAGES * S::STAGE;
  float* s_turn = reinterpret_cast<float*>(after);
  float2* s_col = reinterpret_cast<float2*>(after + EPI_WARPS * TURN);  // [2][BN] {w_scale, bias}
  uint64_t* bars = reinterpret_cast<uint64_t*>(after + EPI_WARPS * TURN + 2 * BN * 8);
  const uint32_t bFull = tc::smem_u32(bars), bEmpty = bFull + 8 * STAGES;
  const uint32_t bAcc = bEmpty + 8 * STAGES, bFree = bAcc + 16;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bars + 24);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 25);
  int* code = reinterpret_cast<int*>(bars + 26);
  static_assert(2 * STAGES + 4 <= 24, "barriers");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_ctarank() : 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      tc::mbar_init(bFull + 8 * s, 2);  // A's and B's issuers
      tc::mbar_init(bEmpty + 8 * s, 1);
    }
    for (int r = 0; r < 2; ++r) {
      tc::mbar_init(bAcc + 8 * r, 1);
      tc::mbar_init(bFree + 8 * r, EPI_WARPS * CG);
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
                   "n"(2 * BN));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       tc::smem_u32((const void*)tmem_slot)),
                   "n"(2 * BN));
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
  const int first = CG == 2 ? (int)tc::cluster_id_x() : (int)blockIdx.x;
  const int step = CG == 2 ? (int)tc::nclusters_x() : (int)gridDim.x;
  // a unit's chunks of k
  auto chunk_range = [&](int unit, int& c0, int& c1) {
    c0 = unit % p.splits * p.chunks_per_split;
    c1 = min(p.chunks, c0 + p.chunks_per_split);
  };
  pdl_wait();

  if (warp < 2) {
    // ============ TMA: warp 0 loads A, warp 1 loads B (both CTAs of a pair) ============
    const bool elected = tc::elect_one(), is_a = warp == 0;
    const CUtensorMap* map = is_a ? &mA : &mB;
    const bool mn = is_a ? AMN : BMN, blocked = is_a ? p.a_blocked : p.b_blocked;
    const int rows = is_a ? 128 : BN / CG, zmul = is_a ? p.az : p.bz;
    const uint32_t bytes = is_a && !AMN ? (uint32_t)p.a_bytes : (uint32_t)(rows * ROW);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int unit = first; unit < p.units && ok; unit += step) {
      const Place pl = place(unit / p.splits, p.tiles_m, p.tiles_n);
      const int at = is_a ? pl.mt * BM + (int)rank * 128 : pl.nt * BN + (int)rank * (BN / CG);
      const int z = pl.g * zmul;
      int c0, c1;
      chunk_range(unit, c0, c1);
      for (int kc = c0; kc < c1; ++kc) {
        if (!tc::mbar_wait(bEmpty + 8 * stage, phase ^ 1u, abort_flag, code, 1)) {
          ok = false;
          break;
        }
        const uint32_t dst = base + stage * S::STAGE + (is_a ? 0 : S::A_BYTES);
        const uint32_t full = lFull + 8 * stage;
        if (elected) {
          // the leader expects both CTAs' bytes; the peer's may land first
          if (rank == 0) tc::mbar_expect_tx(bFull + 8 * stage, CG * bytes);
          if (!mn) {
            load3<CG>(dst, map, full, kc * KE, at, z);
          } else if (blocked) {
            load4<CG>(dst, map, full, 0, kc * KE, at >> 6, z);
          } else {
            for (int i = 0; i < rows / 64; ++i)
              load3<CG>(dst + i * MN_BOX, map, full, at + 64 * i, kc * KE, z);
          }
        }
        if (++stage == STAGES) {
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
      constexpr uint32_t ID = idesc<TYPE>(BM, BN, AMN, BMN);
      // a step further along k, in 16-byte units: 32 bytes of a row, or 16 rows of 128 bytes
      constexpr uint32_t IA = AMN ? 128 : 2, IB = BMN ? 128 : 2;
      int stage = 0, sums = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int unit = first; unit < p.units && ok; unit += step) {
        int c0, c1;
        chunk_range(unit, c0, c1);
        for (int kc = c0; kc < c1 && ok;) {
          const int end = SUMS ? min(c1, kc + SUM_CHUNKS) : c1, r = sums & 1;
          if (sums >= 2 && !tc::mbar_wait(bFree + 8 * r, (uint32_t)(sums / 2 - 1) & 1, abort_flag, code, 2)) {
            ok = false;
            break;
          }
          tc::tc_fence_after();
          const uint32_t d = tmem + (uint32_t)(r * BN);
          for (uint32_t acc = 0; kc < end; ++kc) {
            if (!tc::mbar_wait(bFull + 8 * stage, phase, abort_flag, code, 3)) {
              ok = false;
              break;
            }
            tc::tc_fence_after();
            const uint32_t sA = base + stage * S::STAGE, sB = sA + S::A_BYTES;
            const uint64_t dA = AMN ? tc::sw128_mn_desc(sA, MN_BOX) : tc::sw128_desc(sA);
            const uint64_t dB = BMN ? tc::sw128_mn_desc(sB, MN_BOX) : tc::sw128_desc(sB);
            if (elected) {
#pragma unroll
              for (int i = 0; i < 4; ++i) mma<TYPE, CG>(d, dA + i * IA, dB + i * IB, ID, acc | (uint32_t)i);
              commit<CG>(bEmpty + 8 * stage);
            }
            acc = 1;
            if (++stage == STAGES) {
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
  } else if (warp >= FIRST_EPI) {
    // ============ results ============
    const int ew = warp - FIRST_EPI, q = warp & 3, half = ew >> 2, et = threadIdx.x - 32 * FIRST_EPI;
    float* turn = s_turn + ew * (TURN / 4);
    const Epilogue& e = p.e;
    int sums = 0, tile = 0;
    bool ok = true;
    auto wait_sum = [&]() {
      ok = tc::mbar_wait_warp(bAcc + 8 * (sums & 1), (uint32_t)(sums >> 1) & 1, abort_flag, code, 4);
      tc::tc_fence_after();
      return tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)((sums & 1) * BN + half * HALF);
    };
    auto free_sum = [&]() {
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) tc::mbar_arrive_remote(lFree + 8 * (sums & 1));
        else tc::mbar_arrive(bFree + 8 * (sums & 1));
      }
      ++sums;
    };
    for (int unit = first; unit < p.units; unit += step, ++tile) {
      const Place pl = place(unit / p.splits, p.tiles_m, p.tiles_n);
      const int row0 = pl.mt * BM + (int)rank * 128 + q * 32, rows = p.m - row0;
      const int64_t g = pl.g, row = row0 + lane;
      int c0, c1;
      chunk_range(unit, c0, c1);
      float2* col = s_col + (tile & 1) * BN;
      float xs = 1.f;
      if (FORWARD && !p.part) {
        for (int i = et; i < BN; i += 32 * EPI_WARPS) {
          const int n = pl.nt * BN + i;
          float2 v = make_float2(1.f, 0.f);
          if (n < p.n && e.w_scale.data) v.x = __ldg(e.w_scale.data + g * e.w_scale.group + n);
          if (n < p.n && e.bias.data) v.y = __ldg(e.bias.data + g * e.bias.group + n);
          col[i] = v;
        }
        if (e.x_scale.data && lane < rows) xs = __ldg(e.x_scale.data + g * e.x_scale.group + row);
        asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
      }
      if (!ok) continue;  // (a warp that gave up still comes to the others' barrier)
      // 32 results of this lane's row, from column c of the warp's half
      auto results = [&](float (&u)[32], int c) {
        const int n0 = pl.nt * BN + half * HALF + c, cols = p.n - n0;
        if (rows <= 0 || cols <= 0) return;
        if (p.part) {
          const int64_t o = ((int64_t)(unit % p.splits) * p.groups + g) * p.m + row0;
          store_row<float>(p.part + o * p.ldp + n0, p.ldp, rows, cols, 32, turn, u);
          return;
        }
        if constexpr (FORWARD) {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float2 v = col[half * HALF + c + i];
            u[i] = fmaf(u[i], xs * v.x, v.y);
          }
          if (e.pre.data)
            store_row<bf16>((bf16*)e.pre.data + g * e.pre.group + (int64_t)row0 * e.pre.row + n0,
                            e.pre.row, rows, cols, p.pre_align, turn, u);
          with_act(e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 32; ++i) u[i] = act_value<decltype(act)::value>(u[i], e.slope);
          });
          if (e.residual.data) {
            float v[32];
            load_row<T>((const T*)e.residual.data + g * e.residual.group +
                            (int64_t)row0 * e.residual.row + n0,
                        e.residual.row, rows, cols, p.res_align, turn, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) u[i] += v[i];
          }
        }
        store_row<T>((T*)e.y.data + g * e.y.group + (int64_t)row0 * e.y.row + n0, e.y.row, rows, cols,
                     p.y_align, turn, u);
      };
      if constexpr (SUMS) {
        float acc[HALF];
#pragma unroll
        for (int i = 0; i < HALF; ++i) acc[i] = 0.f;
        for (int kc = c0; kc < c1; kc += SUM_CHUNKS) {
          const uint32_t t = wait_sum();
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < HALF; c += 32) {
            uint32_t r[32];
            LIPZ_TMEM_LD32(t + c, r);
            tc::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c + i] += __uint_as_float(r[i]);
          }
          free_sum();
        }
        if (!ok) continue;
#pragma unroll
        for (int c = 0; c < HALF; c += 32) {
          float u[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) u[i] = acc[c + i];
          results(u, c);
        }
      } else {
        const uint32_t t = wait_sum();
        if (!ok) continue;
#pragma unroll 1
        for (int c = 0; c < HALF; c += 32) {
          uint32_t r[32];
          float u[32];
          LIPZ_TMEM_LD32(t + c, r);
          tc::tmem_wait_ld();
          if (c + 32 == HALF) free_sum();
#pragma unroll
          for (int i = 0; i < 32; ++i) u[i] = __uint_as_float(r[i]);
          results(u, c);
        }
      }
    }
  }
  tc::tc_fence_before();
  if constexpr (CG == 2) tc::cluster_sync_all();
  else __syncthreads();
  tc::tc_fence_after();
  if (warp == 2) {
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * BN));
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * BN));
  }
  if (threadIdx.x == 0 && *code && p.err) *reinterpret_cast<volatile int*>(p.err) = *code;
}

// Sum of the parts of k, in order, and the epilogue. E columns per thread.
struct FinishParams {
  Epilogue e;
  const float* part;
  int64_t ldp, split_stride, total;  // rows of all groups
  int splits, m, n;
};
template <int E>
__global__ void __launch_bounds__(256) k_finish(const FinishParams p) {
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  if (r >= p.total) return;
  const Epilogue& e = p.e;
  for (int64_t c = ((int64_t)blockIdx.y * 32 + (threadIdx.x & 31)) * E; c < p.n;
       c += (int64_t)gridDim.y * 32 * E) {
    const int64_t g = r / p.m, m = r - g * p.m;
    float u[E];
#pragma unroll
    for (int i = 0; i < E; ++i) u[i] = 0.f;
    for (int s = 0; s < p.splits; ++s) {
      const float* q = p.part + s * p.split_stride + r * p.ldp + c;
      if constexpr (E == 4) {
        const float4 v = *reinterpret_cast<const float4*>(q);
        u[0] += v.x, u[1] += v.y, u[2] += v.z, u[3] += v.w;
      } else {
        u[0] += *q;
      }
    }
    const float xs = e.x_scale.data ? e.x_scale.data[g * e.x_scale.group + m] : 1.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (e.w_scale.data) u[i] *= xs * e.w_scale.data[g * e.w_scale.group + c + i];
      if (e.bias.data) u[i] += e.bias.data[g * e.bias.group + c + i];
    }
    auto put = [&](auto t, const lipz_mat& d) {
      using T = decltype(t);
      T* o = (T*)d.data + g * d.group + m * d.row + c;
      if constexpr (E == 1) {
        *o = from_f<T>(u[0]);
      } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(o) = make_float4(u[0], u[1], u[2], u[3]);
      } else {
        *reinterpret_cast<uint2*>(o) = make_uint2(tc::pack_bf16(u[0], u[1]), tc::pack_bf16(u[2], u[3]));
      }
    };
    if (e.pre.data) put(bf16{}, e.pre);
    with_act(e.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < E; ++i) u[i] = act_value<decltype(act)::value>(u[i], e.slope);
    });
    if (e.residual.data) {
      const int64_t o = g * e.residual.group + m * e.residual.row + c;
#pragma unroll
      for (int i = 0; i < E; ++i)
        u[i] += e.y.type == LIPZ_FP32 ? ((const float*)e.residual.data)[o + i]
                                      : __bfloat162float(((const bf16*)e.residual.data)[o + i]);
    }
    if (e.y.type == LIPZ_FP32) put(float{}, e.y);
    else put(bf16{}, e.y);
  }
}

// Rows copied to rows of whole 16-byte units (the bytes past a row's last are zero). A thread forms 16
// bytes of one row.
template <typename U>
__global__ void __launch_bounds__(256)
    k_align_rows(const U* __restrict__ src, int64_t group, int64_t ld, uint4* __restrict__ dst,
                 int64_t rows, int64_t total, int cols, int units) {
  constexpr int E = 16 / sizeof(U);
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  if (r >= total) return;
  const int64_t g = r / rows;
  const U* s = src + g * group + (r - g * rows) * ld;
  for (int u = blockIdx.y * 32 + (threadIdx.x & 31); u < units; u += gridDim.y * 32) {
    union {
      uint4 v;
      U e[E];
    } w;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t c = (int64_t)u * E + i;
      w.e[i] = c < cols ? s[c] : U(0);
    }
    dst[r * units + u] = w.v;
  }
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

struct Plan {
  int cg, bn, splits;
  bool sums;
  int64_t tiles_m, tiles_n, chunks, chunks_per_split, ldp;
  bool copy_a, copy_b;
  int64_t lda, ldb;  // of the copies
  uint64_t a_bytes, b_bytes, part_bytes;
};

Plan make_plan(const Gemm& g) {
  Plan p{};
  const int eb = type_bytes(g.type), unit = 16 / eb;
  const Extent xa = extent(g.a, g.m, g.k), xb = extent(g.b, g.n, g.k);
  p.copy_a = !tma_takes(g.a, xa, g.groups, eb);
  p.copy_b = !tma_takes(g.b, xb, g.groups, eb);
  auto round256 = [](int64_t v) { return (uint64_t)ceil_div(v, 256) * 256; };
  p.lda = ceil_div(xa.cols, unit) * unit;
  p.ldb = ceil_div(xb.cols, unit) * unit;
  p.a_bytes = p.copy_a ? round256(g.groups * xa.rows * p.lda * eb) : 0;
  p.b_bytes = p.copy_b ? round256(g.groups * xb.rows * p.ldb * eb) : 0;
  p.chunks = ceil_div(g.k * eb, ROW);
  p.sums = g.e.y.type == LIPZ_FP32;
  // The shape and the number of parts of k that take the fewest clocks by a model of a unit's time: its
  // MMA steps (pairs of 256 x 256 run at the tensor cores' rate, narrower ones are bound by shared memory)
  // or its epilogue, whichever is longer, and once the ring's and the epilogue's latency; parts of k cost
  // another launch and their way through L2.
  const int sms = sm_count();
  struct Config { int cg, bn; double step, epi; };
  static const Config configs[] = {{2, 256, 128, 5000}, {2, 128, 86, 2600}, {1, 128, 86, 2600}, {1, 64, 60, 1400}};
  double best = 0;
  for (const Config& c : configs) {
    if (p.sums && c.bn > 128) continue;
    const int64_t tm = ceil_div(g.m, 128 * c.cg), tn = ceil_div(g.n, c.bn), tiles = tm * tn * g.groups;
    const int64_t slots = sms / c.cg;
    for (int64_t s = 1; s <= 64 && s <= p.chunks; s *= 2) {
      const int64_t per = ceil_div(p.chunks, s), parts = ceil_div(p.chunks, per);
      if (parts != s && s > 1) continue;
      if (s > 1 && tiles * s > 2 * slots) continue;
      const double mma = per * 4 * c.step, waves = (double)ceil_div(tiles * s, slots);
      double t = waves * (mma > c.epi ? mma : c.epi) + (mma > c.epi ? c.epi : mma) + 2000;
      if (s > 1) t += 5000 + (double)g.groups * g.m * g.n * 4 * s * 2 / 4000;
      if (tiles * s > INT32_MAX) continue;
      if (best == 0 || t < best) {
        best = t;
        p.cg = c.cg, p.bn = c.bn, p.splits = (int)s;
        p.tiles_m = tm, p.tiles_n = tn, p.chunks_per_split = per;
      }
    }
  }
  p.ldp = ceil_div(g.n, 8) * 8;
  p.part_bytes = p.splits > 1 ? round256((int64_t)p.splits * g.groups * g.m * p.ldp * 4) : 0;
  return p;
}

// Sets the kernel's shared memory once per device.
template <typename K>
cudaError_t prepare_kernel(K kernel, int smem, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && done.load() >> dev & 1) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess && dev < 64) done.fetch_or((uint64_t)1 << dev);
  return e;
}

template <int TYPE, int CG, int BN, bool AMN, bool BMN, typename T>
cudaError_t launch(const Gemm& g, const Plan& p, void* part, cudaStream_t st) {
  using S = Shape<CG, BN>;
  CUtensorMap ma, mb;
  GemmParams k{};
  const Extent xa = extent(g.a, g.m, g.k), xb = extent(g.b, g.n, g.k);
  k.a_blocked = AMN && g.m % 64 == 0;
  k.b_blocked = BMN && g.n % 64 == 0;
  const int arows = AMN ? 64 : (int)(g.m >= 128 ? 128 : ceil_div(g.m, 8) * 8);
  const int brows = BMN ? 64 : BN / CG;
  if (!encode(&ma, g.a, xa, g.groups, TYPE, arows, k.a_blocked ? 2 : 0) ||
      !encode(&mb, g.b, xb, g.groups, TYPE, brows, k.b_blocked ? BN / CG / 64 : 0))
    return cudaErrorInvalidValue;
  k.e = g.e;
  k.part = (float*)part;
  k.err = timeout_word();
  k.ldp = p.ldp;
  k.groups = (int)g.groups, k.m = (int)g.m, k.n = (int)g.n;
  k.tiles_m = (int)p.tiles_m, k.tiles_n = (int)p.tiles_n;
  k.splits = p.splits;
  k.units = (int)(p.tiles_m * p.tiles_n * g.groups * p.splits);
  k.chunks = (int)p.chunks, k.chunks_per_split = (int)p.chunks_per_split;
  k.a_bytes = arows * ROW;
  k.az = g.groups > 1 && g.a.group != 0, k.bz = g.groups > 1 && g.b.group != 0;
  auto align = [&](const lipz_mat& m) {
    return !m.data ? 0 : rows_aligned(m, g.groups, g.m, 32) ? 32 : rows_aligned(m, g.groups, g.m, 16) ? 16 : 0;
  };
  k.y_align = align(g.e.y), k.res_align = align(g.e.residual), k.pre_align = align(g.e.pre);
  static std::atomic<uint64_t> done{0};
  auto kernel = k_gemm_op<TYPE, CG, BN, AMN, BMN, T>;
  cudaError_t e = prepare_kernel(kernel, S::SMEM, done);
  if (e != cudaSuccess) return e;
  const int slots = sm_count() / CG, ctas = (k.units < slots ? k.units : slots) * CG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  const bool shared = st == nullptr || st == cudaStreamLegacy || st == cudaStreamPerThread;
  cfg.attrs = attr;
  cfg.numAttrs = shared ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, kernel, ma, mb, k);
}

template <int TYPE, bool AMN, bool BMN>
cudaError_t launch_shape(const Gemm& g, const Plan& p, void* part, cudaStream_t st) {
  if (p.sums) {
    if (p.cg == 2) return launch<TYPE, 2, 128, AMN, BMN, float>(g, p, part, st);
    if (p.bn == 128) return launch<TYPE, 1, 128, AMN, BMN, float>(g, p, part, st);
    return launch<TYPE, 1, 64, AMN, BMN, float>(g, p, part, st);
  }
  if (p.cg == 2 && p.bn == 256) return launch<TYPE, 2, 256, AMN, BMN, bf16>(g, p, part, st);
  if (p.cg == 2) return launch<TYPE, 2, 128, AMN, BMN, bf16>(g, p, part, st);
  if (p.bn == 128) return launch<TYPE, 1, 128, AMN, BMN, bf16>(g, p, part, st);
  return launch<TYPE, 1, 64, AMN, BMN, bf16>(g, p, part, st);
}

cudaError_t align_rows(Operand* o, const Extent& x, int64_t groups, int eb, int64_t ld, void* dst,
                       cudaStream_t st) {
  const int units = (int)(ld * eb / 16);
  const int64_t total = groups * x.rows;
  const dim3 grid = rows_by_columns(total, units);
  cudaError_t e =
      eb == 2 ? launch_pdl(k_align_rows<unsigned short>, grid, dim3(256), 0, st,
                           (const unsigned short*)o->data, o->group, o->ld, (uint4*)dst, x.rows, total,
                           (int)x.cols, units)
              : launch_pdl(k_align_rows<unsigned char>, grid, dim3(256), 0, st,
                           (const unsigned char*)o->data, o->group, o->ld, (uint4*)dst, x.rows, total,
                           (int)x.cols, units);
  o->data = dst;
  o->ld = ld;
  o->group = x.rows * ld;
  return e;
}

}  // namespace

uint64_t gemm_workspace(const Gemm& g) {
  const Plan p = make_plan(g);
  return p.a_bytes + p.b_bytes + p.part_bytes;
}

cudaError_t gemm(const Gemm& args, void* workspace, cudaStream_t st) {
  Gemm g = args;
  const Plan p = make_plan(g);
  const int eb = type_bytes(g.type);
  char* w = (char*)workspace;
  cudaError_t e = cudaSuccess;
  if (p.copy_a) e = align_rows(&g.a, extent(g.a, g.m, g.k), g.groups, eb, p.lda, w, st);
  if (e == cudaSuccess && p.copy_b)
    e = align_rows(&g.b, extent(g.b, g.n, g.k), g.groups, eb, p.ldb, w + p.a_bytes, st);
  if (e != cudaSuccess) return e;
  void* part = p.splits > 1 ? w + p.a_bytes + p.b_bytes : nullptr;
  if (g.type == LIPZ_E4M3) e = launch_shape<LIPZ_E4M3, false, false>(g, p, part, st);
  else if (g.a.k_major && g.b.k_major) e = launch_shape<LIPZ_BF16, false, false>(g, p, part, st);
  else if (g.a.k_major) e = launch_shape<LIPZ_BF16, false, true>(g, p, part, st);
  else e = launch_shape<LIPZ_BF16, true, true>(g, p, part, st);
  if (e != cudaSuccess || !part) return e;
  FinishParams f{g.e, (const float*)part, p.ldp, g.groups * g.m * p.ldp, g.groups * g.m, p.splits,
                 (int)g.m, (int)g.n};
  auto four = [&](const lipz_mat& m) {
    return !m.data || rows_aligned(m, g.groups, g.m, 4 * type_bytes(m.type));
  };
  const bool vec = g.n % 4 == 0 && four(g.e.y) && four(g.e.pre);
  const dim3 grid = rows_by_columns(f.total, vec ? g.n / 4 : g.n);
  return vec ? launch_pdl(k_finish<4>, grid, dim3(256), 0, st, f)
             : launch_pdl(k_finish<1>, grid, dim3(256), 0, st, f);
}

}  // namespace ops
}  // namespace lipz
