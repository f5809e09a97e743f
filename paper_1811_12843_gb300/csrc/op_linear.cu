// Matrix product with bias, activation and residual, and its backward pass: a few rows in a kernel of
// their own, else by the tensor-core product of op_gemm.cu.
#include <type_traits>

#include "op_gemm.h"
#include "ops.cuh"

namespace lipz {
namespace ops {

namespace {

// y for a few rows: w's rows stream through the warps of a block, W_ROWS at a time, each warp over its part
// of k (parts > 1: few columns), and meet the rows of x, which stay in L1. Bound: HBM (w is read once).
constexpr int W_ROWS = 4, VEC_WARPS = 4;

// 16 bytes of a row (VEC), or one element.
template <int TYPE>
struct Elem {
  typedef typename std::conditional<TYPE == LIPZ_BF16, bf16, e4m3>::type T;
  static constexpr int E = 16 / sizeof(T);
  template <bool VEC>
  struct Vec {
    uint32_t w[VEC ? 4 : 1];
    __device__ __forceinline__ void zero() {
#pragma unroll
      for (uint32_t& v : w) v = 0;
    }
    __device__ __forceinline__ void load(const T* p) {
      if constexpr (VEC) {
        const uint4 r = __ldg(reinterpret_cast<const uint4*>(p));
        w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
      } else if constexpr (TYPE == LIPZ_BF16) {
        w[0] = __ldg(reinterpret_cast<const unsigned short*>(p));
      } else {
        w[0] = __ldg(p);
      }
    }
    __device__ __forceinline__ void decode(float* v) const {
      if constexpr (TYPE == LIPZ_BF16) {
#pragma unroll
        for (int i = 0; i < (VEC ? 8 : 1); ++i)
          v[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
      } else {
#pragma unroll
        for (int i = 0; i < (VEC ? 8 : 1); ++i) {
          const __half2_raw h =
              __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (i & 1) * 16), __NV_E4M3);
          const float2 f = __half22float2(__half2(h));
          v[2 * i] = f.x;
          if constexpr (VEC) v[2 * i + 1] = f.y;
        }
      }
    }
  };
};

struct VecParams {
  lipz_mat x, w;
  Epilogue e;
  int64_t n, k;
  int rows, parts;  // warps that share an output
};

// KEPT: u is kept as a checkpoint: VEC_WARPS * parts warps, so that a block has 16 outputs. (Up to 512 threads have 128
// registers each; four rows in whole vectors spill 56 bytes there, over 8 bits 160.)
template <int TYPE, int R, bool VEC, bool KEPT>
__global__ void __launch_bounds__(32 * VEC_WARPS * (KEPT ? VEC_WARPS : 1)) k_linear_rows(const VecParams p) {
  using L = Elem<TYPE>;
  using T = typename L::T;
  constexpr int E = VEC ? L::E : 1;
  __shared__ float s[VEC_WARPS * (KEPT ? VEC_WARPS : 1)][R * W_ROWS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % p.parts;
  const int per_block = KEPT ? VEC_WARPS * W_ROWS : VEC_WARPS / p.parts * W_ROWS;
  static_assert(VEC_WARPS * W_ROWS == LIPZ_BLOCK, "a block of a checkpoint");
  const int64_t g = blockIdx.y, n0 = (int64_t)blockIdx.x * per_block + warp / p.parts * W_ROWS;
  const T* x = (const T*)p.x.data + g * p.x.group;
  const T* w = (const T*)p.w.data + g * p.w.group;
  pdl_wait();
  float acc[W_ROWS][R];
#pragma unroll
  for (int j = 0; j < W_ROWS; ++j)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[j][r] = 0.f;
  const int64_t units = p.k / E, step = 32 * p.parts;
  int64_t wo[W_ROWS], xo[R];
#pragma unroll
  for (int j = 0; j < W_ROWS; ++j) wo[j] = min(n0 + j, p.n - 1) * p.w.row;
#pragma unroll
  for (int r = 0; r < R; ++r) xo[r] = (int64_t)min(r, p.rows - 1) * p.x.row;
  // AHEAD vectors of each of w's rows are in flight while those before them are multiplied. Measured at 1 x
  // 8192 -> 8192 (134 MB, 19.8 us at the copy rate): 28.7 us; two rows and four vectors 38.9, and 38.9
  // without those ahead.
  constexpr int AHEAD = 2;
  if (n0 < p.n) {
    typename L::template Vec<VEC> next[AHEAD][W_ROWS], wv[AHEAD][W_ROWS];
    auto bring = [&](int64_t u0) {
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
#pragma unroll
        for (int j = 0; j < W_ROWS; ++j) {
          const int64_t u = u0 + a * step;
          next[a][j].zero();
          if (u < units) next[a][j].load(w + wo[j] + u * E);
        }
    };
    bring(part * 32 + lane);
    for (int64_t u0 = part * 32 + lane; u0 < units; u0 += AHEAD * step) {
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
#pragma unroll
        for (int j = 0; j < W_ROWS; ++j) wv[a][j] = next[a][j];
      bring(u0 + AHEAD * step);
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        const int64_t u = u0 + a * step;
        if (u >= units) break;
        float wf[W_ROWS][E];
#pragma unroll
        for (int j = 0; j < W_ROWS; ++j) wv[a][j].decode(wf[j]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          typename L::template Vec<VEC> xv;
          float xf[E];
          xv.load(x + xo[r] + u * E);
          xv.decode(xf);
#pragma unroll
          for (int j = 0; j < W_ROWS; ++j)
#pragma unroll
            for (int i = 0; i < E; ++i) acc[j][r] = fmaf(wf[j][i], xf[i], acc[j][r]);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < W_ROWS; ++j)
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int o = 16; o; o >>= 1) acc[j][r] += __shfl_xor_sync(0xffffffffu, acc[j][r], o);
      if (lane == 0) s[warp][r * W_ROWS + j] = acc[j][r];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < per_block * p.rows; i += blockDim.x) {
    const int c = i % per_block, r = i / per_block;
    const int64_t n = (int64_t)blockIdx.x * per_block + c;
    if (n >= p.n && !KEPT) continue;
    float u = 0.f;
    for (int q = 0; q < p.parts; ++q) u += s[c / W_ROWS * p.parts + q][r * W_ROWS + c % W_ROWS];
    if constexpr (KEPT) finish_kept(p.e, g, r, n, n < p.n, u);
    else finish(p.e, g, r, n, u);
  }
}

// Whether rows of x and w are whole 16-byte units.
bool in_units(const lipz_linear_args& a) {
  return a.k % (16 / type_bytes(a.x.type)) == 0 && rows_aligned(a.x, a.groups, a.rows, 16) &&
         rows_aligned(a.w, a.groups, a.n, 16);
}

// Few rows go to k_linear_rows while it is the faster. Beside w's bytes it pays for each row of x that meets
// them, so the weights that it takes fall with the square of the rows, and for each block, so the outputs of
// all groups are bounded; element by element (rows off the 16-byte grid) its rate is bounded by the loads,
// and the tensor cores' product has such rows copied first. There and on the tensor cores, us, bf16 (between events,
// a launch with them, after a flush of L2; among other calls 1 x 4096 -> 4096 takes 10.2):
//   rows   1 x 4096 -> 4096 12.3, 16.8   2 x 4096 -> 4096 14.4, 16.6   4 x 4096 -> 4096 19.7, 16.4
//          1 x 8192 -> 8192 29.1, 34.8   2 x 8192 -> 8192 42.0, 34.4   4 x 1024 -> 1024  8.2, 14.3
//   blocks 1 x 512 -> 16384 11.1, 12.0   1 x 512 -> 32768 14.6, 14.3   1 x 256 -> 512, 256 groups 35.5, 18.8
//   odd    2 x 1001 -> 8001 19.1, 23.4   2 x 4001 -> 8001 58.6, 52.2   1 x 777 -> 500, 16 groups 15.6, 19.6
bool few_rows(const lipz_linear_args& a) {
  if (a.rows > 4) return false;
  const double work = (double)a.rows * a.rows * a.groups * a.n * a.k;
  if (!in_units(a)) return work <= 32 << 20;
  return (a.rows == 1 || work <= 64 << 20) && a.groups * a.n <= 12 << 10;
}

template <int TYPE, bool VEC, bool KEPT>
cudaError_t launch_rows(const VecParams& p, dim3 grid, cudaStream_t st) {
  const dim3 block(32 * VEC_WARPS * (KEPT ? p.parts : 1));
  if (p.rows == 1) return launch_pdl(k_linear_rows<TYPE, 1, VEC, KEPT>, grid, block, 0, st, p);
  if (p.rows == 2) return launch_pdl(k_linear_rows<TYPE, 2, VEC, KEPT>, grid, block, 0, st, p);
  return launch_pdl(k_linear_rows<TYPE, 4, VEC, KEPT>, grid, block, 0, st, p);
}
template <int TYPE>
cudaError_t launch_rows(const VecParams& p, bool vec, dim3 grid, cudaStream_t st) {
  if (p.e.kept.data)
    return vec ? launch_rows<TYPE, true, true>(p, grid, st) : launch_rows<TYPE, false, true>(p, grid, st);
  return vec ? launch_rows<TYPE, true, false>(p, grid, st) : launch_rows<TYPE, false, false>(p, grid, st);
}

cudaError_t linear_rows(const lipz_linear_args& a, const Epilogue& e, cudaStream_t st) {
  const int per = 16 / type_bytes(a.x.type);
  const bool vec = in_units(a);
  // warps share an output where whole rows would leave the SMs with fewer than eight warps each
  int parts = 1;
  while (parts < VEC_WARPS && a.groups * ceil_div(a.n, W_ROWS) * parts < 8 * sm_count() &&
         a.k >= (vec ? per : 1) * 64 * parts)
    parts *= 2;
  const VecParams p{a.x, a.w, e, a.n, a.k, (int)a.rows, parts};
  const int outputs = VEC_WARPS / (e.kept.data ? 1 : parts) * W_ROWS;
  const dim3 grid((unsigned)ceil_div(a.n, outputs), (unsigned)a.groups);
  return a.x.type == LIPZ_E4M3 ? launch_rows<LIPZ_E4M3>(p, vec, grid, st) : launch_rows<LIPZ_BF16>(p, vec, grid, st);
}

Epilogue epilogue_of(const lipz_linear_args& a, const lipz_blocks& kept) {
  Epilogue e{a.y, a.residual, a.pre, a.x_scale, a.w_scale, a.bias, a.act, a.slope, kept};
  if (a.x.type != LIPZ_E4M3) e.x_scale.data = e.w_scale.data = nullptr;
  return e;
}
Products product_of(const lipz_linear_args& a, const lipz_blocks& kept) {
  return {{{{a.x.data, a.x.group, a.x.row, true}, {a.w.data, a.w.group, a.w.row, true}, a.x.type,
            a.groups, a.rows, a.n, a.k, epilogue_of(a, kept)}},
          1};
}

// du = dy act'(pre), in bf16 rows of ldu elements, and the sums of its columns over the block's rows:
// 32 vectors of columns by 8 rows at a time; the blocks after those copy operands' rows. Bound: HBM.
struct DuArgs {
  lipz_mat dy, pre;
  lipz_blocks kept;  // in pre's place, or data null
  bf16* du;     // [groups][rows][ldu], or null: the sums only
  float* part;  // [groups][row_blocks][n], or null: no sums
  int64_t rows, n, ldu, rows_per_block;
  int act;
  float slope;
  int col_blocks, row_blocks, blocks;  // of a group; of all groups
};

// ALIGNED: rows of whole 16-byte units; else 8 columns are brought from the aligned words that hold them
// (777 x 1001 with the copies beside it: one at a time 8.6 us, so 7.9, most of it latency).
// KEPT: pre is a checkpoint, whose multiples are widened and multiplied by their power two at a time; four blocks to an SM,
// a row at a time, which needs no more registers than those have (8192 x 4096, gelu, the sums alone: 36.0 us; four rows
// at a time 37.5 with spills, 37.6 with three blocks; of five or six blocks, which are no whole waves, 46).
// COPIES: rows of checkpoints may be among those copied.
template <bool ALIGNED, bool KEPT, bool COPIES>
__global__ void __launch_bounds__(256, KEPT ? 4 : 0) k_du(const DuArgs p, const __grid_constant__ CopyJobs jobs) {
  constexpr int E = 8;
  __shared__ float s[8][32 * E + 1];
  pdl_wait();
  if ((int)blockIdx.x >= p.blocks) return copy_rows<COPIES>(jobs, (int)blockIdx.x - p.blocks);
  const int per = p.col_blocks * p.row_blocks, in_group = blockIdx.x % per;
  const int row_block = in_group / p.col_blocks, col_block = in_group - row_block * p.col_blocks;
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int64_t c = ((int64_t)col_block * 32 + tx) * E, g = blockIdx.x / per;
  const int64_t r0 = row_block * p.rows_per_block;
  const int64_t r1 = min(p.rows, r0 + p.rows_per_block);
  auto load = [&](const lipz_mat& m, int64_t r, float* v) {
    const bf16* src = (const bf16*)m.data + g * m.group + r * m.row + c;
    if constexpr (ALIGNED) {
      load_vec<bf16, E>(src, v);
    } else {
      const uint4 w = bytes16((const uint8_t*)src, (p.n - c) * 2);  // (columns past the last are zero)
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = __uint_as_float(e & 1 ? ww[e >> 1] & 0xFFFF0000u : ww[e >> 1] << 16);
    }
  };
  auto load_kept = [&](int64_t r, float* v) {
    const int8_t* src = p.kept.data + g * p.kept.group + r * p.kept.row + c;
    const float unit = block_unit(__ldg(p.kept.scale + g * p.kept.scale_group + r * p.kept.scale_row + (c >> 4)));
    uint2 w;
    if constexpr (ALIGNED) {
      w = __ldg(reinterpret_cast<const uint2*>(src));
    } else {
      const uint4 b = bytes16((const uint8_t*)src, min(p.n - c, (int64_t)E));
      w = make_uint2(b.x, b.y);
    }
    block_values(w.x, unit, v);
    block_values(w.y, unit, v + 4);
  };
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  with_act(p.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if (c < p.n) {
#pragma unroll (KEPT ? 1 : 4)
      for (int64_t r = r0 + ty; r < r1; r += 8) {
        float d[E];
        load(p.dy, r, d);
        if constexpr (ACT != LIPZ_ACT_NONE) {
          float u[E];
          if constexpr (KEPT) {
            load_kept(r, u);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              const float2 both = unpack2(mul2(pack2(d[e], d[e + 1]), act_slope_pair<ACT>(pack2(u[e], u[e + 1]), p.slope)));
              d[e] = both.x, d[e + 1] = both.y;
            }
          } else {
            load(p.pre, r, u);
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= act_slope<ACT>(u[e], p.slope);
          }
        }
        if (p.du) store_vec<bf16, E>(p.du + (g * p.rows + r) * p.ldu + c, d);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += d[e];
      }
    }
  });
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < E; ++e) s[ty][tx * E + e] = sum[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * E; i += 256) {
    const int64_t col = (int64_t)col_block * 32 * E + i;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) v += s[q][i];
    if (col < p.n) p.part[(g * p.row_blocks + row_block) * p.n + col] = v;
  }
}

// The workspace of a backward call: du (where dy is not it), the parts of db, then the products' own. dx and
// dw share a launch where their results are bf16 and neither's sums are long.
struct BackPlan {
  bool vec, need_du;
  int64_t ldu, blocks, rows_per_block;
  uint64_t du_bytes, db_bytes, bytes;
  int launches;
  Products q[2];
  GemmPlan plan[2];
};
// kept_x, kept_pre: checkpoints in the places of x and pre, or data null.
BackPlan back_plan(const lipz_linear_backward_args& a, const lipz_blocks& kept_x, const lipz_blocks& kept_pre) {
  BackPlan b{};
  b.vec = a.n % 8 == 0 && rows_aligned(a.dy, a.groups, a.rows, 16) &&
          (kept_pre.data ? rows_aligned(bytes_of(kept_pre), a.groups, a.rows, 8)
                         : !a.pre.data || rows_aligned(a.pre, a.groups, a.rows, 16));
  // Without an activation du is dy: written where the products cannot read dy itself, unless one of them is
  // all that is wanted. (Instead of a copy for each: 8192 x 4096 -> 4097 401 -> 357 us, 144 groups of 100 x
  // 256 -> 501 55 -> 45.)
  const bool readable = rows_aligned(a.dy, a.groups, a.rows, 16) && (a.rows <= 1 || a.dy.row >= a.n);
  const bool both_or_db = a.db.data ? a.dx.data || a.dw.data : a.dx.data && a.dw.data;
  b.need_du = a.act != LIPZ_ACT_NONE ? a.dx.data || a.dw.data : !readable && both_or_db;
  b.ldu = ceil_div(a.n, 8) * 8;
  if (a.groups == 0 || a.rows == 0) return b;
  // enough blocks to fill the device, of 8 rows or more
  const int64_t cols = ceil_div(a.n, 256), fill = 8 * sm_count();
  const int64_t want = ceil_div(fill, cols * a.groups);
  b.rows_per_block = ceil_div(ceil_div(a.rows, want), 8) * 8;
  b.blocks = ceil_div(a.rows, b.rows_per_block);
  auto round256 = [](int64_t v) { return (uint64_t)ceil_div(v, 256) * 256; };
  b.du_bytes = b.need_du ? round256(a.groups * a.rows * b.ldu * 2) : 0;
  b.db_bytes = a.db.data ? round256(a.groups * b.blocks * a.n * 4) : 0;
  b.bytes = b.du_bytes + b.db_bytes;
  const void* d = b.need_du ? a.workspace : a.dy.data;
  const int64_t dg = b.need_du ? a.rows * b.ldu : a.dy.group, dr = b.need_du ? b.ldu : a.dy.row;
  const Gemm dx{{d, dg, dr, true}, {a.w.data, a.w.group, a.w.row, false}, LIPZ_BF16, a.groups, a.rows,
                a.k, a.n, {a.dx}};
  Operand x{a.x.data, a.x.group, a.x.row, false};
  if (kept_x.data)
    x = {kept_x.data, kept_x.group, kept_x.row, false, kept_x.scale, kept_x.scale_group, kept_x.scale_row};
  const Gemm dw{{d, dg, dr, false}, x, LIPZ_BF16, a.groups, a.n, a.k, a.rows, {a.dw}};
  // bf16 results run as planned for both, whether or not both are asked for, so that one's values do not
  // depend on the other; fp32 results are planned by themselves, and so are products of which one is so long
  // that its shape would slow the other (16392 x 4096 -> 4096: 708 us in one launch, 662 in two)
  Products both{{dx, dw}, 2};
  both.g[0].e.y.type = both.g[1].e.y.type = LIPZ_BF16;
  const GemmPlan joint = plan_products(both);
  auto add = [&](const Gemm& g, int i) {
    if (!g.e.y.data) return;
    if (g.e.y.type == LIPZ_FP32 || joint.sums) {
      b.q[b.launches] = {{g}, 1};
      b.plan[b.launches] = plan_products(b.q[b.launches]);
      ++b.launches;
      return;
    }
    if (!b.launches || b.q[b.launches - 1].g[0].e.y.type == LIPZ_FP32) {
      b.plan[b.launches] = joint;
      b.q[b.launches++].n = 0;
    }
    Products& q = b.q[b.launches - 1];
    b.plan[b.launches - 1].p[q.n] = joint.p[i];
    q.g[q.n++] = g;
    plan_space(q, &b.plan[b.launches - 1]);
  };
  add(dx, 0);
  add(dw, 1);
  for (int i = 0; i < b.launches; ++i) b.bytes += b.plan[i].bytes;
  return b;
}

}  // namespace

uint64_t linear_workspace(const lipz_linear_args& a, const lipz_blocks& kept) {
  return a.groups == 0 || a.rows == 0 || few_rows(a) ? 0 : plan_products(product_of(a, kept)).bytes;
}

cudaError_t linear(const lipz_linear_args& a, const lipz_blocks& kept, cudaStream_t st, uint64_t* need) {
  *need = 0;
  if (a.groups == 0 || a.rows == 0) return cudaSuccess;
  if (few_rows(a)) return linear_rows(a, epilogue_of(a, kept), st);
  Products q = product_of(a, kept);
  const GemmPlan plan = plan_products(q);
  *need = plan.bytes;
  if (!space_given(a.workspace, a.workspace_bytes, *need)) return cudaSuccess;
  RowCopy copies[4];
  const int n = plan_copies(plan, &q, a.workspace, copies);
  const cudaError_t e = run_copies(copy_jobs(copies, n), st);
  return e != cudaSuccess ? e : run_products(plan, q, a.workspace, nullptr, st);
}

uint64_t linear_backward_workspace(const lipz_linear_backward_args& a, const lipz_blocks& kept_x,
                                   const lipz_blocks& kept_pre) {
  return back_plan(a, kept_x, kept_pre).bytes;
}

cudaError_t linear_backward(const lipz_linear_backward_args& a, const lipz_blocks& kept_x,
                            const lipz_blocks& kept_pre, cudaStream_t st, uint64_t* need) {
  *need = 0;
  if (a.groups == 0) return cudaSuccess;
  if (a.rows == 0) {  // sums over no rows
    cudaError_t e = cudaSuccess;
    const int64_t row_bytes = a.k * type_bytes(a.dw.type);
    for (int64_t g = 0; g < a.groups && e == cudaSuccess; ++g) {
      if (a.dw.data)
        e = cudaMemset2DAsync((char*)a.dw.data + g * a.dw.group * type_bytes(a.dw.type),
                              a.n > 1 ? a.dw.row * type_bytes(a.dw.type) : row_bytes, 0, row_bytes,
                              a.n, st);
      if (a.db.data && e == cudaSuccess)
        e = cudaMemsetAsync(a.db.data + g * a.db.group, 0, a.n * 4, st);
    }
    return e;
  }
  BackPlan b = back_plan(a, kept_x, kept_pre);
  *need = b.bytes;
  if (!space_given(a.workspace, a.workspace_bytes, *need)) return cudaSuccess;
  bf16* du = b.need_du ? (bf16*)a.workspace : nullptr;
  float* part = a.db.data ? (float*)((char*)a.workspace + b.du_bytes) : nullptr;
  char* rest = (char*)a.workspace + b.du_bytes + b.db_bytes;
  RowCopy copies[4];
  int n = 0;
  char* at[2] = {rest, rest + b.plan[0].bytes};
  for (int i = 0; i < b.launches; ++i) n += plan_copies(b.plan[i], &b.q[i], at[i], copies + n);
  const CopyJobs jobs = copy_jobs(copies, n);
  cudaError_t e;
  if (du || part) {
    const int64_t cols = ceil_div(a.n, 256), blocks = cols * b.blocks * a.groups;
    const DuArgs p{a.dy, a.pre, kept_pre, du, part, a.rows, a.n, b.ldu, b.rows_per_block, a.act, a.slope,
                   (int)cols, (int)b.blocks, (int)blocks};
    const dim3 grid((unsigned)(blocks + jobs.blocks));
    auto run = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(256), 0, st, p, jobs); };
    if (kept_pre.data) e = b.vec ? run(k_du<true, true, true>) : run(k_du<false, true, true>);
    else if (jobs.kept) e = b.vec ? run(k_du<true, false, true>) : run(k_du<false, false, true>);
    else e = b.vec ? run(k_du<true, false, false>) : run(k_du<false, false, false>);
  } else {
    e = run_copies(jobs, st);
  }
  const PartSums sums{part, a.n, (int)a.groups, (int)b.blocks, a.db};
  if (e == cudaSuccess && part && !b.launches)
    e = sum_parts(part, a.groups, (int)b.blocks, a.n, a.db, SUM_WAYS, st);
  for (int i = 0; i < b.launches && e == cudaSuccess; ++i)
    e = run_products(b.plan[i], b.q[i], at[i], i == 0 && part ? &sums : nullptr, st);
  return e;
}

}  // namespace ops
}  // namespace lipz
