// C ABI of the residual-block operators: every argument that the host can check is checked here, then
// the kernels of op_norm.cu, op_linear.cu and op_gemm.cu are launched.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <utility>

#include "op_gemm.h"

using namespace lipz;

namespace lipz {
namespace ops {

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 152;
  }
  return n;
}

// A word of pinned memory for each host thread, which every device reaches: the kernels of the thread's calls store
// to it, and the thread reads it without waiting for them. Words stay with the process, since a kernel, or a graph
// that was captured from a call, may outlive the thread.
thread_local int* t_word = nullptr;

int* timeout_word() {
  if (t_word) return t_word;
  constexpr int BLOCK = 1024;
  static std::mutex mutex;
  static int* block = nullptr;
  static int used = BLOCK;
  const std::lock_guard<std::mutex> lock(mutex);
  if (used == BLOCK) {
    // (allocating host memory is not part of a graph that another thread's stream may be capturing)
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    cudaThreadExchangeStreamCaptureMode(&mode);
    int* p = nullptr;
    const cudaError_t e = cudaHostAlloc((void**)&p, BLOCK * sizeof(int), cudaHostAllocPortable | cudaHostAllocMapped);
    cudaThreadExchangeStreamCaptureMode(&mode);
    if (e != cudaSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    memset(p, 0, BLOCK * sizeof(int));
    block = p;
    used = 0;
  }
  return t_word = block + used++;
}

}  // namespace ops
}  // namespace lipz

namespace {

thread_local char t_error[256];

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(t_error, sizeof t_error, fmt, ap);
  va_end(ap);
  return code;
}

int finish(const char* call, cudaError_t e) {
  if (e == cudaSuccess) return LIPZ_OK;
  cudaGetLastError();
  return fail(LIPZ_ERR_CUDA, "%s: %s", call, cudaGetErrorString(e));
}

// Whether a kernel of this thread's calls gave up on a wait since the last report.
int take_timeout(const char* call) {
  int* const word = ops::t_word;  // (null: no kernel has been given one)
  const int code = word ? __atomic_exchange_n(word, 0, __ATOMIC_ACQ_REL) : 0;
  if (!code) return LIPZ_OK;
  return fail(LIPZ_ERR_TIMEOUT,
              "%s: an earlier call's kernel gave up on a wait (%d): its results are not valid", call, code);
}

constexpr int64_t MAX_EXTENT = INT32_MAX;

// One call's checks: the first failure stays.
struct Check {
  const char* call;
  int64_t groups, rows;
  int rc = LIPZ_OK;

  bool want(bool ok, const char* what) {
    if (!ok && rc == LIPZ_OK) rc = fail(LIPZ_ERR_INVALID, "%s: %s", call, what);
    return ok && rc == LIPZ_OK;
  }
  bool extent(int64_t v, int64_t lo, int64_t hi, const char* name) {
    if ((v < lo || v > hi) && rc == LIPZ_OK)
      rc = fail(LIPZ_ERR_INVALID, "%s: %s must be in %lld..%lld (got %lld)", call, name, (long long)lo,
                (long long)hi, (long long)v);
    return rc == LIPZ_OK;
  }
  bool extents() {
    return extent(groups, 0, 65535, "groups") && extent(rows, 0, MAX_EXTENT, "rows") &&
           want(groups * rows <= MAX_EXTENT, "groups x rows must stay below 2^31");
  }
  void fail_mat(const char* name, const char* what) {
    if (rc == LIPZ_OK) rc = fail(LIPZ_ERR_INVALID, "%s: %s %s", call, name, what);
  }
  // types: a set of 1 << type. Outputs' rows and groups may not overlap.
  bool mat(const lipz_mat& m, const char* name, int64_t nrows, int64_t cols, int types, bool out,
           bool optional = false) {
    if (rc != LIPZ_OK) return false;
    if (!m.data) {
      if (!optional && groups > 0 && nrows > 0) fail_mat(name, "is null");
      return rc == LIPZ_OK;
    }
    if (m.type < 0 || m.type > 2 || !(types >> m.type & 1))
      fail_mat(name, "has a type that this call does not take");
    else if ((uintptr_t)m.data % ops::type_bytes(m.type)) fail_mat(name, "is not aligned to its type");
    else if (nrows > 1 && (m.row < (out ? cols : 0))) fail_mat(name, "has a row stride that is too small");
    else if (groups > 1 && m.group < 0) fail_mat(name, "has a negative group stride");
    else if (out && groups > 1 && nrows > 0) {
      // one group inside the other's row gaps is not looked for: groups lie apart, or rows interleave
      const int64_t span = (nrows - 1) * m.row + cols;
      const bool apart = m.group >= span, woven = m.group >= cols && m.row >= (groups - 1) * m.group + cols;
      if (!apart && !(woven || nrows == 1 && m.group >= cols)) fail_mat(name, "has groups that overlap");
    }
    return rc == LIPZ_OK;
  }
  bool vec(const lipz_vec& v, const char* name, int64_t n, bool out, bool optional = false) {
    if (rc != LIPZ_OK) return false;
    if (!v.data) {
      if (!optional && groups > 0 && n > 0) fail_mat(name, "is null");
    } else if ((uintptr_t)v.data % 4) fail_mat(name, "is not aligned to its type");
    else if (groups > 1 && v.group < (out ? n : 0)) fail_mat(name, "has a group stride that is too small");
    return rc == LIPZ_OK;
  }
  bool space(const void* p, uint64_t have, uint64_t need) {
    if (rc != LIPZ_OK || ops::space_given(p, have, need)) return rc == LIPZ_OK;
    if (!p || have < need)
      rc = fail(LIPZ_ERR_INVALID, "%s: the workspace must hold %llu bytes", call, (unsigned long long)need);
    else
      rc = fail(LIPZ_ERR_INVALID, "%s: the workspace must be 256-byte aligned", call);
    return rc == LIPZ_OK;
  }
};

constexpr int F32 = 1 << LIPZ_FP32, B16 = 1 << LIPZ_BF16, F8 = 1 << LIPZ_E4M3;

template <typename A>
bool struct_ok(const A* a, const char* call, int* rc) {
  if (a && a->struct_size == sizeof(A)) return true;
  *rc = fail(LIPZ_ERR_INVALID, a ? "%s: struct_size does not match the library" : "%s: null arguments", call);
  return false;
}

int check(const lipz_rmsnorm_args* a) {
  Check c{"lipz_rmsnorm"};
  if (!struct_ok(a, c.call, &c.rc)) return c.rc;
  c.groups = a->groups, c.rows = a->rows;
  if (!c.extents() || !c.extent(a->dim, 1, LIPZ_NORM_MAX_DIM, "dim")) return c.rc;
  c.want(a->eps >= 0.f, "eps must not be negative");
  c.mat(a->x, "x", a->rows, a->dim, F32 | B16, false);
  const int t = 1 << a->x.type;
  c.mat(a->residual, "residual", a->rows, a->dim, t, false, true);
  c.mat(a->sum, "sum", a->rows, a->dim, t, true, true);
  c.mat(a->y, "y", a->rows, a->dim, t | F8, true);
  c.vec(a->weight, "weight", a->dim, false);
  if (a->y.data && a->y.type == LIPZ_E4M3) c.vec(a->scale, "scale", a->rows, true);
  c.vec(a->rstd, "rstd", a->rows, true, true);
  return c.rc;
}

int check(const lipz_rmsnorm_backward_args* a) {
  Check c{"lipz_rmsnorm_backward"};
  if (!struct_ok(a, c.call, &c.rc)) return c.rc;
  c.groups = a->groups, c.rows = a->rows;
  if (!c.extents() || !c.extent(a->dim, 1, LIPZ_NORM_MAX_DIM, "dim")) return c.rc;
  c.mat(a->dy, "dy", a->rows, a->dim, F32 | B16, false);
  const int t = 1 << a->dy.type;
  c.mat(a->s, "s", a->rows, a->dim, t, false);
  c.mat(a->dsum, "dsum", a->rows, a->dim, t, false, true);
  c.mat(a->dx, "dx", a->rows, a->dim, t, true);
  c.vec(a->weight, "weight", a->dim, false);
  c.vec(a->rstd, "rstd", a->rows, false);
  c.vec(a->dweight, "dweight", a->dim, true, true);
  return c.rc;
}

uint64_t space_of(const lipz_rmsnorm_backward_args& a) {
  const int parts = ops::rmsnorm_backward_parts(a);
  return parts > 1 && a.dweight.data ? (uint64_t)a.groups * parts * a.dim * 4 : 0;
}

int check(const lipz_quantize_rows_args* a) {
  Check c{"lipz_quantize_rows"};
  if (!struct_ok(a, c.call, &c.rc)) return c.rc;
  c.groups = a->groups, c.rows = a->rows;
  if (!c.extents() || !c.extent(a->dim, 1, MAX_EXTENT, "dim")) return c.rc;
  c.mat(a->x, "x", a->rows, a->dim, F32 | B16, false);
  c.mat(a->q, "q", a->rows, a->dim, F8, true);
  c.vec(a->scale, "scale", a->rows, true);
  return c.rc;
}

int check(const lipz_linear_args* a) {
  Check c{"lipz_linear"};
  if (!struct_ok(a, c.call, &c.rc)) return c.rc;
  c.groups = a->groups, c.rows = a->rows;
  if (!c.extents() || !c.extent(a->k, 1, MAX_EXTENT, "k") || !c.extent(a->n, 1, MAX_EXTENT, "n") ||
      !c.want(a->groups * a->n <= MAX_EXTENT, "groups x n must stay below 2^31"))
    return c.rc;
  c.extent(a->act, LIPZ_ACT_NONE, LIPZ_ACT_SILU, "act");
  c.mat(a->x, "x", a->rows, a->k, B16 | F8, false);
  c.mat(a->w, "w", a->n, a->k, 1 << a->x.type, false);
  c.mat(a->y, "y", a->rows, a->n, B16 | F32, true);
  c.mat(a->residual, "residual", a->rows, a->n, 1 << a->y.type, false, true);
  c.mat(a->pre, "pre", a->rows, a->n, B16, true, true);
  if (a->x.type == LIPZ_E4M3) {
    c.vec(a->x_scale, "x_scale", a->rows, false);
    c.vec(a->w_scale, "w_scale", a->n, false);
  }
  c.vec(a->bias, "bias", a->n, false, true);
  return c.rc;
}

int check(const lipz_linear_backward_args* a) {
  Check c{"lipz_linear_backward"};
  if (!struct_ok(a, c.call, &c.rc)) return c.rc;
  c.groups = a->groups, c.rows = a->rows;
  if (!c.extents() || !c.extent(a->k, 1, MAX_EXTENT, "k") || !c.extent(a->n, 1, MAX_EXTENT, "n") ||
      !c.want(a->groups * a->n <= MAX_EXTENT, "groups x n must stay below 2^31"))
    return c.rc;
  c.extent(a->act, LIPZ_ACT_NONE, LIPZ_ACT_SILU, "act");
  c.mat(a->dy, "dy", a->rows, a->n, B16, false);
  c.mat(a->x, "x", a->rows, a->k, B16, false, !a->dw.data);
  c.mat(a->w, "w", a->n, a->k, B16, false, !a->dx.data);
  c.mat(a->pre, "pre", a->rows, a->n, B16, false, a->act == LIPZ_ACT_NONE);
  c.mat(a->dx, "dx", a->rows, a->k, B16 | F32, true, true);
  c.mat(a->dw, "dw", a->n, a->k, B16 | F32, true, true);
  c.vec(a->db, "db", a->n, true, true);
  return c.rc;
}

// ---- outputs that share memory with other arguments: a kernel would read what it has already overwritten

// `groups` times `rows` rows of `width` bytes, `group` and `row` bytes apart.
struct Region {
  uintptr_t at;
  int64_t width, rows, row, groups, group;

  // (strides of 0 repeat one row or group)
  static Region of(const void* data, int64_t width, int64_t rows, int64_t row, int64_t groups, int64_t group) {
    if (!data || rows <= 0 || groups <= 0) return {0, 0, 0, 0, 0, 0};
    const bool many = rows > 1 && row, grouped = groups > 1 && group;
    return {(uintptr_t)data, width, many ? rows : 1, many ? row : 0, grouped ? groups : 1, grouped ? group : 0};
  }
  bool same_place(const Region& o) const {
    return at == o.at && width == o.width && rows == o.rows && row == o.row && groups == o.groups && group == o.group;
  }
  int64_t span() const { return (rows - 1) * row + (groups - 1) * group + width; }
  // Rows or groups without gaps between them as one row.
  Region joined() const {
    Region r = *this;
    for (int i = 0; i < 2; ++i) {
      if (r.rows > 1 && r.row == r.width) r.width *= r.rows, r.rows = 1, r.row = 0;
      if (r.groups > 1 && r.group == r.width) r.width *= r.groups, r.groups = 1, r.group = 0;
    }
    return r;
  }
};

int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }

// Whether some byte certainly lies in both. Exact where the two have one row stride and one group stride (rows or
// groups that lie without gaps count as one row, which goes with any stride); of others only their starts are
// compared.
bool meet(const Region& p, const Region& q) {
  if (!p.width || !q.width) return false;
  if (q.at >= p.at + p.span() || p.at >= q.at + q.span()) return false;
  const Region a = p.joined(), b = q.joined();
  if ((a.rows > 1 && b.rows > 1 && a.row != b.row) || (a.groups > 1 && b.groups > 1 && a.group != b.group))
    return a.at == b.at;
  // rows i apart and groups j apart meet if -b.width < d - i row - j group < a.width
  struct Steps {
    int64_t by, lo, hi;
  } outer{a.groups > 1 ? a.group : b.group, 1 - b.groups, a.groups - 1},
      inner{a.rows > 1 ? a.row : b.row, 1 - b.rows, a.rows - 1};
  if (outer.by < inner.by) std::swap(outer, inner);
  const int64_t d = (int64_t)(b.at - a.at);
  // the steps (from lo to hi) whose multiple lies in [x0, x1]
  auto within = [](Steps s, int64_t x0, int64_t x1) {
    if (s.lo == s.hi) return x0 <= 0 && 0 <= x1 ? s : Steps{0, 1, 0};
    return Steps{s.by, std::max(s.lo, -floor_div(-x0, s.by)), std::min(s.hi, floor_div(x1, s.by))};
  };
  const Steps o = within(outer, d - inner.hi * inner.by - a.width + 1, d - inner.lo * inner.by + b.width - 1);
  // (a few, unless rows lie across one another as only an input's may)
  for (int64_t j = o.lo; j <= o.hi && j - o.lo < 64; ++j) {
    const int64_t rest = d - j * outer.by;
    const Steps i = within(inner, rest - a.width + 1, rest + b.width - 1);
    if (i.lo <= i.hi) return true;
  }
  return false;
}

// One call's outputs against its inputs and one another.
struct Overlap {
  const char* call;
  int64_t groups;
  struct Part {
    const char* name;
    Region r;
    unsigned places;  // of an output: the inputs whose own place it may have
  };
  Part in[6], out[4];
  int ins = 0, outs = 0;

  Overlap(const char* call_, int64_t groups_) : call(call_), groups(groups_) {}
  Region region(const lipz_mat& m, int64_t rows, int64_t cols) const {
    const int64_t b = ops::type_bytes(m.type);
    return Region::of(m.data, cols * b, rows, m.row * b, groups, m.group * b);
  }
  Region region(const lipz_vec& v, int64_t n) const { return Region::of(v.data, n * 4, 1, 0, groups, v.group * 4); }
  unsigned input(const char* name, const lipz_mat& m, int64_t rows, int64_t cols) {
    in[ins] = {name, region(m, rows, cols), 0u};
    return 1u << ins++;
  }
  void input(const char* name, const lipz_vec& v, int64_t n) { in[ins++] = {name, region(v, n), 0u}; }
  void output(const char* name, const lipz_mat& m, int64_t rows, int64_t cols, unsigned places = 0) {
    out[outs++] = {name, region(m, rows, cols), places};
  }
  void output(const char* name, const lipz_vec& v, int64_t n) { out[outs++] = {name, region(v, n), 0u}; }

  int result() const {
    for (int i = 0; i < outs; ++i) {
      for (int j = 0; j < ins; ++j)
        if (meet(out[i].r, in[j].r) && !(out[i].places >> j & 1 && out[i].r.same_place(in[j].r)))
          return fail(LIPZ_ERR_INVALID, "%s: %s overlaps %s", call, out[i].name, in[j].name);
      for (int j = 0; j < i; ++j)
        if (meet(out[i].r, out[j].r))
          return fail(LIPZ_ERR_INVALID, "%s: %s overlaps %s", call, out[i].name, out[j].name);
    }
    return LIPZ_OK;
  }
};

// (The row operators' threads have an element of every input in registers before they write one there.)
int overlap(const lipz_rmsnorm_args& a) {
  Overlap o{"lipz_rmsnorm", a.groups};
  const unsigned own = o.input("x", a.x, a.rows, a.dim) | o.input("residual", a.residual, a.rows, a.dim);
  o.input("weight", a.weight, a.dim);
  o.output("sum", a.sum, a.rows, a.dim, own);
  o.output("y", a.y, a.rows, a.dim, own);
  if (a.y.type == LIPZ_E4M3) o.output("scale", a.scale, a.rows);
  o.output("rstd", a.rstd, a.rows);
  return o.result();
}
int overlap(const lipz_rmsnorm_backward_args& a) {
  Overlap o{"lipz_rmsnorm_backward", a.groups};
  const unsigned own = o.input("dy", a.dy, a.rows, a.dim) | o.input("s", a.s, a.rows, a.dim) |
                       o.input("dsum", a.dsum, a.rows, a.dim);
  o.input("weight", a.weight, a.dim);
  o.input("rstd", a.rstd, a.rows);
  o.output("dx", a.dx, a.rows, a.dim, own);
  o.output("dweight", a.dweight, a.dim);
  return o.result();
}
int overlap(const lipz_quantize_rows_args& a) {
  Overlap o{"lipz_quantize_rows", a.groups};
  o.input("x", a.x, a.rows, a.dim);
  o.output("q", a.q, a.rows, a.dim);
  o.output("scale", a.scale, a.rows);
  return o.result();
}
int overlap(const lipz_linear_args& a) {
  Overlap o{"lipz_linear", a.groups};
  const unsigned own = o.input("residual", a.residual, a.rows, a.n);
  o.input("x", a.x, a.rows, a.k);
  o.input("w", a.w, a.n, a.k);
  o.input("bias", a.bias, a.n);
  if (a.x.type == LIPZ_E4M3) {
    o.input("x_scale", a.x_scale, a.rows);
    o.input("w_scale", a.w_scale, a.n);
  }
  o.output("y", a.y, a.rows, a.n, own);
  o.output("pre", a.pre, a.rows, a.n);
  return o.result();
}
int overlap(const lipz_linear_backward_args& a) {
  Overlap o{"lipz_linear_backward", a.groups};
  o.input("dy", a.dy, a.rows, a.n);
  if (a.dw.data) o.input("x", a.x, a.rows, a.k);
  if (a.dx.data) o.input("w", a.w, a.n, a.k);
  if (a.act != LIPZ_ACT_NONE) o.input("pre", a.pre, a.rows, a.n);
  o.output("dx", a.dx, a.rows, a.k);
  o.output("dw", a.dw, a.n, a.k);
  o.output("db", a.db, a.n);
  return o.result();
}

}  // namespace

extern "C" {

int lipz_rmsnorm(const lipz_rmsnorm_args* a, void* stream) {
  if (int rc = check(a)) return rc;
  if (int rc = overlap(*a)) return rc;
  if (int rc = take_timeout("lipz_rmsnorm")) return rc;
  return finish("lipz_rmsnorm", ops::rmsnorm(*a, (cudaStream_t)stream));
}

int lipz_rmsnorm_backward_workspace(const lipz_rmsnorm_backward_args* a, uint64_t* bytes) {
  if (int rc = check(a)) return rc;
  if (!bytes) return fail(LIPZ_ERR_INVALID, "lipz_rmsnorm_backward_workspace: bytes is null");
  *bytes = space_of(*a);
  return LIPZ_OK;
}

int lipz_rmsnorm_backward(const lipz_rmsnorm_backward_args* a, void* stream) {
  if (int rc = check(a)) return rc;
  Check c{"lipz_rmsnorm_backward", a->groups, a->rows};
  if (!c.space(a->workspace, a->workspace_bytes, space_of(*a))) return c.rc;
  if (int rc = overlap(*a)) return rc;
  if (int rc = take_timeout(c.call)) return rc;
  return finish(c.call, ops::rmsnorm_backward(*a, (cudaStream_t)stream));
}

int lipz_quantize_rows(const lipz_quantize_rows_args* a, void* stream) {
  if (int rc = check(a)) return rc;
  if (int rc = overlap(*a)) return rc;
  if (int rc = take_timeout("lipz_quantize_rows")) return rc;
  return finish("lipz_quantize_rows", ops::quantize_rows(*a, (cudaStream_t)stream));
}

int lipz_linear_workspace(const lipz_linear_args* a, uint64_t* bytes) {
  if (int rc = check(a)) return rc;
  if (!bytes) return fail(LIPZ_ERR_INVALID, "lipz_linear_workspace: bytes is null");
  *bytes = ops::linear_workspace(*a);
  return LIPZ_OK;
}

int lipz_linear(const lipz_linear_args* a, void* stream) {
  if (int rc = check(a)) return rc;
  Check c{"lipz_linear", a->groups, a->rows};
  if (int rc = overlap(*a))
    return c.space(a->workspace, a->workspace_bytes, ops::linear_workspace(*a)) ? rc : c.rc;
  if (int rc = take_timeout(c.call)) return rc;
  uint64_t need;
  const cudaError_t e = ops::linear(*a, (cudaStream_t)stream, &need);
  if (!c.space(a->workspace, a->workspace_bytes, need)) return c.rc;
  return finish(c.call, e);
}

int lipz_linear_backward_workspace(const lipz_linear_backward_args* a, uint64_t* bytes) {
  if (int rc = check(a)) return rc;
  if (!bytes) return fail(LIPZ_ERR_INVALID, "lipz_linear_backward_workspace: bytes is null");
  *bytes = ops::linear_backward_workspace(*a);
  return LIPZ_OK;
}

int lipz_linear_backward(const lipz_linear_backward_args* a, void* stream) {
  if (int rc = check(a)) return rc;
  Check c{"lipz_linear_backward", a->groups, a->rows};
  if (int rc = overlap(*a))
    return c.space(a->workspace, a->workspace_bytes, ops::linear_backward_workspace(*a)) ? rc : c.rc;
  if (int rc = take_timeout(c.call)) return rc;
  uint64_t need;
  const cudaError_t e = ops::linear_backward(*a, (cudaStream_t)stream, &need);
  if (!c.space(a->workspace, a->workspace_bytes, need)) return c.rc;
  return finish(c.call, e);
}

int lipz_operator_status(void) { return take_timeout("lipz_operator_status"); }

const char* lipz_operator_error(void) { return t_error; }

}  // extern "C"
