// Plans and launches of the tensor-core products (op_gemm_kernel.cuh).
#include "op_gemm_kernel.cuh"

namespace lipz {
namespace ops {

namespace {

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

template <bool KEPT>
__global__ void __launch_bounds__(256) k_copy_rows(const __grid_constant__ CopyJobs jobs) {
  pdl_wait();
  copy_rows<KEPT>(jobs, blockIdx.x);
}

// Blocks of 8 rows by 32 columns' threads; columns past 65535 blocks are looped over.
dim3 rows_by_columns(int64_t rows, int64_t columns) {
  const int64_t y = ceil_div(columns, 32);
  return dim3((unsigned)ceil_div(rows, 8), (unsigned)(y < 65535 ? y : 65535));
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
  const bool kept = g0.e.kept.data;
  const int64_t long_chunks = kept ? KEPT_MIN : LONG_CHUNKS;
  auto kept_sums = [&](int64_t chunks) {
    const int64_t quarter = ceil_div(chunks, 4), most = fp32 ? SUM_CHUNKS : KEPT_MAX;
    const int64_t n = quarter < KEPT_MIN ? KEPT_MIN : quarter < most ? quarter : most;
    return (double)ceil_div(chunks, n);
  };
  const bool by_tma = results_by_tma(g0);
  const bool forward = g0.a.k_major && g0.b.k_major;
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
        t.sums = t.sums || o.chunks_per_split > long_chunks;
        fits = fits && tiles * o.splits <= INT32_MAX / 2 &&
               (o.splits == 1 || tiles * o.splits <= (forward ? 1 : 2) * slots) &&
               (!forward || o.splits == s0);
        const double mma = o.chunks_per_split * 4 * c.step * (eb == 1 ? 1.16 : 1);
        double epi = c.epi + (heavy ? c.act : 0) + (res ? c.residual : 0);
        // A checkpoint beside them: its own stores, and its sums' way into registers, priced as sums of a quarter of the
        // part; in 256-wide tiles, where the MMAs are ahead by two sums, three eighths of their time. (8192 x 1024 ->
        // 4096 66 us by 256 x 128, 92 by 256 x 256; 8192 x 4096 -> 8192 398 and 323, 4100 x 8192 -> 4096 228 and 178.)
        // Prices fitted to such times, not counts of the sums that run (SumChunks): by those all of the latter went to
        // 256 x 128, and small products to parts of k (519 x 1408 -> 128 over 8-bit operands 6.8 us, so 9.5).
        if (kept) epi += c.bn * (c.bn == 256 ? 10 : 3) + kept_sums(o.chunks_per_split) * (c.bn == 256 ? 2700. : 1300.);
        if (kept && c.bn == 256) epi += 0.375 * mma;
        const double unit = mma > epi ? mma : epi;
        work += unit * tiles * o.splits;
        if (unit > top) top = unit;
        if (mma + epi > last) last = mma + epi;
        if (o.splits > 1 && !forward) extra += (double)g.groups * g.m * g.n * 4 * o.splits * 2 / 3000;
        split = split || o.splits > 1;
      }
      // (sums in 256-wide tiles: bf16 results of a checkpoint's product, and of those no others)
      if (!fits || (s0 > 1 && !split) || (c.bn > 128 && t.sums != kept)) continue;
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
      t.direct = true, t.sums = fp32 || o.chunks > long_chunks, t.cg = 1, t.bn = 64;
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
      const int from = t.scale ? 1 : eb;  // bytes of an element
      copies[n++] = {(const uint8_t*)t.data, w, t.group * from, t.ld * from, x.rows, groups * x.rows,
                     x.cols * from, ld * eb / 16, t.scale, t.scale_group, t.scale_ld, 32};
      if (t.scale)
        while (copies[n - 1].lanes > 1 && copies[n - 1].lanes >= copies[n - 1].units) copies[n - 1].lanes /= 2;
      t.data = w, t.ld = ld, t.group = groups > 1 ? x.rows * ld : 0, t.scale = nullptr;
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
    jobs.kept = jobs.kept || c[i].scale;
    jobs.blocks += ceil_div(c[i].total, COPY_ROWS * 32 / c[i].lanes);
  }
  return jobs;
}

cudaError_t run_copies(const CopyJobs& jobs, cudaStream_t st) {
  if (jobs.blocks == 0) return cudaSuccess;
  return launch_pdl(jobs.kept ? k_copy_rows<true> : k_copy_rows<false>, dim3((unsigned)jobs.blocks), dim3(256), 0, st,
                    jobs);
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
  if (g0.e.kept.data) e = run_kept_product(plan, q, st);
  else if (g0.type == LIPZ_E4M3) e = launch_shape<LIPZ_E4M3, true, 0>(q, plan, parts, sums, st);
  else if (g0.a.k_major && g0.b.k_major) e = launch_shape<LIPZ_BF16, true, 0>(q, plan, parts, sums, st);
  else e = launch_shape<LIPZ_BF16, false, 0>(q, plan, parts, sums, st);
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
