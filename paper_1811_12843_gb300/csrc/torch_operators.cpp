// The residual-block operators on torch tensors: checks of a call's tensors, its outputs and workspace from
// torch's allocator, and the library's call on the current stream. Python keeps the signatures and their
// documentation (operators.py). Written against torch's C++ interface because next to kernels of a few
// microseconds the same steps in Python took most of a call: the norm of one row of 4096 to 8 bits 17 us, now 6.5 to
// 8 with two microseconds of kernel, 37 x 1000 -> 500 over 8-bit operands 18.5, now 7.6, the backward of 777 x 500 ->
// 1001 38, now 16. (One guard to a call, results made without torch's dispatcher where nothing listens to it: the
// layer norm that keeps a checkpoint and makes six results 14.5 us, now 9.2.)
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <ATen/record_function.h>
#include <c10/core/InferenceMode.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <string>

#include "lipz.h"

namespace {

using at::ScalarType;
using at::Tensor;

PyObject* g_error;  // LipzError

struct Refusal {
  int code;
  std::string what;
};

constexpr ScalarType F32 = ScalarType::Float, BF16 = ScalarType::BFloat16, E4M3 = ScalarType::Float8_e4m3fn;

int type_of(ScalarType t) { return t == F32 ? LIPZ_FP32 : t == BF16 ? LIPZ_BF16 : t == E4M3 ? LIPZ_E4M3 : -1; }
constexpr int bit(int type) { return 1 << type; }
constexpr int WIDE = bit(LIPZ_FP32) | bit(LIPZ_BF16), HALF = bit(LIPZ_BF16);

struct Shape {
  int dims;
  int64_t d[3];
  Shape(int64_t a) : dims(1), d{a} {}
  Shape(int64_t a, int64_t b) : dims(2), d{a, b} {}
  Shape(int64_t a, int64_t b, int64_t c) : dims(3), d{a, b, c} {}
  bool is(at::IntArrayRef s) const {
    if ((int)s.size() != dims) return false;
    for (int i = 0; i < dims; ++i)
      if (s[i] != d[i]) return false;
    return true;
  }
};

std::string text(at::IntArrayRef s) {
  std::string r = "[";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + "]";
}

// One call: its name, the device of its first tensor (the current one until its end), and the sizes that the others go
// by.
struct Call {
  const char* name;
  int device = -1;
  std::optional<c10::cuda::CUDAGuard> guard;
  bool grouped = false;
  int64_t groups = 1, rows = 0, cols = 0;

  [[noreturn]] void refuse(const std::string& what) const {
    throw Refusal{LIPZ_ERR_INVALID, std::string(name) + ": " + what};
  }
  const Tensor& tensor(PyObject* o, const char* what) const {
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a CUDA tensor");
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided) refuse(std::string(what) + " must be a CUDA tensor");
    // (no call records a graph: its results would have no gradient, without a word)
    if (t.requires_grad() && at::GradMode::is_enabled())
      refuse(std::string(what) + " requires a gradient, and this call records none: use torch.no_grad() or detach()");
    return t;
  }
  static bool adjacent(const Tensor& t) {
    return t.stride(-1) == 1 || t.size(-1) <= 1 || t.numel() == 0;
  }
  lipz_mat view(const Tensor& t, const char* what, int types, bool out = false) const {
    const int type = type_of(t.scalar_type());
    if (type < 0 || !(types >> type & 1))
      refuse(std::string(what) + " has dtype " + at::toString(t.scalar_type()) + ", which is not taken");
    if (!adjacent(t)) refuse(std::string(what) + ": columns must be adjacent");
    const auto st = t.strides();
    void* const data = out ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr());
    return {data, st.size() == 3 ? st[0] : 0, st[st.size() - 2], type, 0};
  }
  // The tensor that gives the call its device, groups, rows and columns.
  lipz_mat first(PyObject* o, const char* what, int types) {
    const Tensor& t = tensor(o, what);
    first(t, what);
    return view(t, what, types);
  }
  void first(const Tensor& t, const char* what) {
    const auto s = t.sizes();
    if (s.size() != 2 && s.size() != 3)
      refuse(std::string(what) + " must be [rows, columns] or [groups, rows, columns]");
    grouped = s.size() == 3;
    if (grouped) groups = s[0];
    rows = s[s.size() - 2], cols = s[s.size() - 1];
    device = t.get_device();
    guard.emplace((c10::DeviceIndex)device);
  }
  const Tensor& like(PyObject* o, const char* what, const Shape& shape) const {
    const Tensor& t = tensor(o, what);
    if (t.get_device() != device)
      refuse(std::string(what) + " must be a CUDA tensor on the same device as the others");
    if (!shape.is(t.sizes()))
      refuse(std::string(what) + " has shape " + text(t.sizes()) + ", not " +
             text(at::IntArrayRef(shape.d, shape.dims)));
    return t;
  }
  Shape matrix(int64_t r, int64_t c) const { return grouped ? Shape(groups, r, c) : Shape(r, c); }
  Shape vector(int64_t n) const { return grouped ? Shape(groups, n) : Shape(n); }
  // A tensor of the caller's that the call writes to; wrote() follows the call. (A copy-on-write clone gets memory
  // of its own here, so an input that may be the same tensor is taken after it.)
  lipz_mat target(PyObject* o, const char* what, int64_t r, int64_t c, int types) const {
    const Tensor& t = like(o, what, matrix(r, c));
    if (t.is_inference() && !c10::InferenceMode::is_enabled())
      refuse(std::string(what) + " is an inference tensor, which is written in inference mode alone");
    return view(t, what, types, true);
  }
  // What autograd has saved of the tensor is no longer what it holds.
  static void wrote(PyObject* o) {
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
  // (None: null)
  lipz_mat mat(PyObject* o, const char* what, int64_t r, int64_t c, int types) const {
    if (o == Py_None) return {};
    return view(like(o, what, matrix(r, c)), what, types);
  }
  lipz_vec vec(PyObject* o, const char* what, int64_t n) const {
    if (o == Py_None) return {};
    const Tensor& t = like(o, what, vector(n));
    if (t.scalar_type() != F32)
      refuse(std::string(what) + " has dtype " + at::toString(t.scalar_type()) + ", taken is torch.float32");
    if (!adjacent(t)) refuse(std::string(what) + ": columns must be adjacent");
    return {(float*)t.const_data_ptr(), grouped ? t.stride(0) : 0};
  }
  // Whether an allocation goes through torch's dispatcher: a dispatch mode or a transform of this thread's, or the
  // profiler, is to see it, or memory is to be filled. Else the same tensor comes from the allocator itself (the layer
  // norm with a checkpoint: 14.5 us of the host by the dispatcher, so 9.2).
  static bool dispatched() {
    const auto keys = c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set;
    const auto& context = at::globalContext();
    return !keys.empty() || at::getStepCallbacksUnlessEmpty(at::RecordScope::FUNCTION).has_value() ||
           (context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory());
  }
  at::TensorOptions options(ScalarType t) const {
    return at::TensorOptions().dtype(t).device(c10::kCUDA, (c10::DeviceIndex)device);
  }
  Tensor empty(const Shape& s, ScalarType t) const {
    const at::IntArrayRef size(s.d, s.dims);
    if (dispatched()) return at::empty(size, options(t));
    return Tensor(at::detail::empty_generic(size, c10::cuda::CUDACachingAllocator::get(),
                                            c10::DispatchKeySet(c10::DispatchKey::CUDA), t, std::nullopt));
  }
  lipz_mat fresh(Tensor& t, int64_t r, int64_t c, ScalarType type) const {
    t = empty(matrix(r, c), type);
    return {t.mutable_data_ptr(), r * c, c, type_of(type), 0};
  }
  lipz_vec fresh(Tensor& t, int64_t n) const {
    t = empty(vector(n), F32);
    return {(float*)t.mutable_data_ptr(), n};
  }
  // A checkpoint: a tuple of its data and its scales.
  static bool is_checkpoint(PyObject* o) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2; }
  lipz_blocks blocks_of(const Tensor& q, const Tensor& s, const std::string& what) const {
    if (q.scalar_type() != ScalarType::Char || s.scalar_type() != ScalarType::Byte)
      refuse(what + ": a checkpoint is of torch.int8, and its scale of torch.uint8");
    if (!adjacent(q) || !adjacent(s)) refuse(what + ": columns must be adjacent");
    const auto a = q.strides(), b = s.strides();
    return {(int8_t*)q.const_data_ptr(), a.size() == 3 ? a[0] : 0, a[a.size() - 2],
            (uint8_t*)s.const_data_ptr(), b.size() == 3 ? b[0] : 0, b[b.size() - 2]};
  }
  lipz_blocks blocks(PyObject* o, const char* what, int64_t r, int64_t c) const {
    const std::string scale = std::string(what) + "'s scale";
    const Tensor& q = like(PyTuple_GET_ITEM(o, 0), what, matrix(r, c));
    return blocks_of(q, like(PyTuple_GET_ITEM(o, 1), scale.c_str(), matrix(r, (c + LIPZ_BLOCK - 1) / LIPZ_BLOCK)),
                     what);
  }
  // Rows begin whole blocks apart.
  lipz_blocks fresh(Tensor& q, Tensor& s, int64_t r, int64_t c) const {
    const int64_t n = (c + LIPZ_BLOCK - 1) / LIPZ_BLOCK, row = n * LIPZ_BLOCK;
    const int64_t size[3] = {groups, r, c}, stride[3] = {r * row, row, 1};
    const int skip = grouped ? 0 : 1;
    const at::IntArrayRef sizes(size + skip, 3 - skip), strides(stride + skip, 3 - skip);
    q = dispatched() ? at::empty_strided(sizes, strides, options(ScalarType::Char))
                     : Tensor(at::detail::empty_strided_generic(sizes, strides, c10::cuda::CUDACachingAllocator::get(),
                                                                c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                                ScalarType::Char));
    s = empty(matrix(r, n), ScalarType::Byte);
    return {(int8_t*)q.mutable_data_ptr(), r * row, row, (uint8_t*)s.mutable_data_ptr(), r * n, n};
  }
  void require(PyObject* o, const char* what) const {
    if (o == Py_None) refuse(std::string(what) + " must be given");
  }
  ScalarType result_type(PyObject* o, const char* what) const {
    const ScalarType t = THPDtype_Check(o) ? ((THPDtype*)o)->scalar_type : ScalarType::Undefined;
    if (t != BF16 && t != F32) refuse(std::string(what) + " must be bfloat16 or float32");
    return t;
  }
  void* stream() const { return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

void done(int rc) {
  if (rc) throw Refusal{rc, lipz_operator_error()};
}

// The library's call on the device's current stream, with the GIL released.
template <typename A>
void run(const Call& c, int (*f)(const A*, void*), const A& a) {
  void* const stream = c.stream();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f(&a, stream);
  Py_END_ALLOW_THREADS
  done(rc);
}
// With the workspace that it asks for, which w takes.
template <typename A, typename W>
void run(const Call& c, int (*query)(const A*, uint64_t*), int (*f)(const A*, void*), A& a, W& w) {
  uint64_t need = 0;
  done(query(&a, &need));
  Tensor space;
  if (need) {
    space = c.empty(Shape((int64_t)need), ScalarType::Byte);
    w.workspace = space.mutable_data_ptr();
    w.workspace_bytes = need;
  }
  run(c, f, a);
}
template <typename A>
void run(const Call& c, int (*query)(const A*, uint64_t*), int (*f)(const A*, void*), A& a) {
  run(c, query, f, a, a);
}

PyObject* give(const Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
PyObject* given(PyObject* o) {
  Py_INCREF(o);
  return o;
}
// A tuple of new references.
template <typename... P>
PyObject* results(P... p) {
  PyObject* const all[] = {p...};
  PyObject* r = PyTuple_New(sizeof...(p));
  for (size_t i = 0; i < sizeof...(p); ++i) {
    if (r && all[i]) PyTuple_SET_ITEM(r, i, all[i]);
    else Py_XDECREF(all[i]);
    if (!all[i]) Py_CLEAR(r);
  }
  return r;
}

// A checkpoint's two tensors (undefined: None).
PyObject* give(const Tensor& q, const Tensor& s) {
  if (!q.defined()) Py_RETURN_NONE;
  return results(give(q), give(s));
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v;
}
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}

// keep: false, true, or "int8" (2)
int keep_of(const Call& c, PyObject* o) {
  if (!PyUnicode_Check(o)) return truth(o);
  if (PyUnicode_CompareWithASCIIString(o, "int8")) c.refuse("keep must be False, True or \"int8\"");
  return 2;
}
// Of a call that keeps nothing in 8 bits: a word would be taken for True, and what it asks for left out.
bool keep_plain(const Call& c, PyObject* o) {
  if (PyUnicode_Check(o)) c.refuse("keep must be False or True: nothing is kept in 8 bits here");
  return truth(o);
}

// x, weight, residual, eps, e4m3, keep, sum_out -> y, sum, scale, rstd
PyObject* rmsnorm(PyObject* const* o) {
  Call c{"rmsnorm"};
  const bool keep = keep_plain(c, o[5]);
  lipz_rmsnorm_args a{};
  a.struct_size = sizeof a;
  a.x = c.first(o[0], "x", WIDE);
  c.require(o[1], "weight");
  a.weight = c.vec(o[1], "weight", c.cols);
  a.eps = number(o[3]);
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  const bool e4m3 = truth(o[4]), own_sum = o[6] != Py_None;
  const ScalarType type = a.x.type == LIPZ_FP32 ? F32 : BF16;
  Tensor y, sum, scale, rstd;
  if (o[2] == Py_None) {
    if (own_sum) c.refuse("sum_out needs a residual");
  } else {
    if (own_sum) {
      a.sum = c.target(o[6], "sum_out", c.rows, c.cols, bit(a.x.type));
      a.x = c.view(c.tensor(o[0], "x"), "x", WIDE);  // (x may be sum_out)
    } else {
      a.sum = c.fresh(sum, c.rows, c.cols, type);
    }
    a.residual = c.mat(o[2], "residual", c.rows, c.cols, bit(a.x.type));
  }
  a.y = c.fresh(y, c.rows, c.cols, e4m3 ? E4M3 : type);
  if (e4m3) a.scale = c.fresh(scale, c.rows);
  if (keep) a.rstd = c.fresh(rstd, c.rows);
  run(c, lipz_rmsnorm, a);
  if (own_sum) c.wrote(o[6]);
  return results(give(y), sum.defined() ? give(sum) : given(own_sum ? o[6] : o[0]), give(scale), give(rstd));
}

// dy, s, rstd, weight, dsum, want_dweight -> dx, dweight
PyObject* rmsnorm_backward(PyObject* const* o) {
  Call c{"rmsnorm_backward"};
  lipz_rmsnorm_backward_args a{};
  a.struct_size = sizeof a;
  a.s = c.first(o[1], "s", WIDE);
  c.require(o[0], "dy"), c.require(o[2], "rstd"), c.require(o[3], "weight");
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  a.dy = c.mat(o[0], "dy", c.rows, c.cols, bit(a.s.type));
  a.rstd = c.vec(o[2], "rstd", c.rows);
  a.weight = c.vec(o[3], "weight", c.cols);
  a.dsum = c.mat(o[4], "dsum", c.rows, c.cols, bit(a.s.type));
  Tensor dx, dweight;
  a.dx = c.fresh(dx, c.rows, c.cols, a.s.type == LIPZ_FP32 ? F32 : BF16);
  if (truth(o[5])) a.dweight = c.fresh(dweight, c.cols);
  run(c, lipz_rmsnorm_backward_workspace, lipz_rmsnorm_backward, a);
  return results(give(dx), give(dweight));
}

// x, weight, bias, residual, eps, e4m3, keep, sum_out -> y, sum, scale, mean, rstd, kept
PyObject* layernorm(PyObject* const* o) {
  Call c{"layernorm"};
  lipz_layernorm_args a{};
  a.struct_size = sizeof a;
  a.x = c.first(o[0], "x", WIDE);
  c.require(o[1], "weight");
  a.weight = c.vec(o[1], "weight", c.cols);
  a.bias = c.vec(o[2], "bias", c.cols);
  a.eps = number(o[4]);
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  const bool e4m3 = truth(o[5]), own_sum = o[7] != Py_None;
  const int keep = keep_of(c, o[6]);
  const ScalarType type = a.x.type == LIPZ_FP32 ? F32 : BF16;
  Tensor y, sum, scale, mean, rstd, q, blocks;
  if (o[3] == Py_None) {
    if (own_sum) c.refuse("sum_out needs a residual");
  } else {
    if (own_sum) {
      a.sum = c.target(o[7], "sum_out", c.rows, c.cols, bit(a.x.type));
      a.x = c.view(c.tensor(o[0], "x"), "x", WIDE);  // (x may be sum_out)
    } else {
      a.sum = c.fresh(sum, c.rows, c.cols, type);
    }
    a.residual = c.mat(o[3], "residual", c.rows, c.cols, bit(a.x.type));
  }
  a.y = c.fresh(y, c.rows, c.cols, e4m3 ? E4M3 : type);
  if (e4m3) a.scale = c.fresh(scale, c.rows);
  if (keep) a.mean = c.fresh(mean, c.rows), a.rstd = c.fresh(rstd, c.rows);
  if (keep == 2) a.kept = c.fresh(q, blocks, c.rows, c.cols);
  run(c, lipz_layernorm, a);
  if (own_sum) c.wrote(o[7]);
  return results(give(y), sum.defined() ? give(sum) : given(own_sum ? o[7] : o[0]), give(scale), give(mean),
                 give(rstd), give(q, blocks));
}

// dy, s, mean, rstd, weight, dsum, want_dweight, want_dbias -> dx, dweight, dbias
PyObject* layernorm_backward(PyObject* const* o) {
  Call c{"layernorm_backward"};
  lipz_layernorm_backward_args a{};
  a.struct_size = sizeof a;
  a.dy = c.first(o[0], "dy", WIDE);
  c.require(o[2], "mean"), c.require(o[3], "rstd"), c.require(o[4], "weight");
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  if (c.is_checkpoint(o[1])) {
    a.kept = c.blocks(o[1], "s", c.rows, c.cols);
  } else {
    c.require(o[1], "s");
    a.s = c.mat(o[1], "s", c.rows, c.cols, bit(a.dy.type));
  }
  a.mean = c.vec(o[2], "mean", c.rows);
  a.rstd = c.vec(o[3], "rstd", c.rows);
  a.weight = c.vec(o[4], "weight", c.cols);
  a.dsum = c.mat(o[5], "dsum", c.rows, c.cols, bit(a.dy.type));
  Tensor dx, dweight, dbias;
  a.dx = c.fresh(dx, c.rows, c.cols, a.dy.type == LIPZ_FP32 ? F32 : BF16);
  if (truth(o[6])) a.dweight = c.fresh(dweight, c.cols);
  if (truth(o[7])) a.dbias = c.fresh(dbias, c.cols);
  run(c, lipz_layernorm_backward_workspace, lipz_layernorm_backward, a);
  return results(give(dx), give(dweight), give(dbias));
}

// x -> data, scale
PyObject* checkpoint_rows(PyObject* const* o) {
  Call c{"checkpoint_rows"};
  lipz_checkpoint_rows_args a{};
  a.struct_size = sizeof a;
  a.x = c.first(o[0], "x", WIDE);
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  Tensor q, blocks;
  a.c = c.fresh(q, blocks, c.rows, c.cols);
  run(c, lipz_checkpoint_rows, a);
  return give(q, blocks);
}

// checkpoint, act's code, slope, out_dtype -> y
PyObject* restore_rows(PyObject* const* o) {
  Call c{"restore_rows"};
  lipz_restore_rows_args a{};
  a.struct_size = sizeof a;
  if (!c.is_checkpoint(o[0])) c.refuse("a checkpoint is taken: its data and its scale");
  const Tensor& q = c.tensor(PyTuple_GET_ITEM(o[0], 0), "the checkpoint");
  c.first(q, "the checkpoint");
  a.c = c.blocks(o[0], "the checkpoint", c.rows, c.cols);
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  a.act = (int)PyLong_AsLong(o[1]);
  a.slope = number(o[2]);
  Tensor y;
  a.y = c.fresh(y, c.rows, c.cols, c.result_type(o[3], "out_dtype"));
  run(c, lipz_restore_rows, a);
  return give(y);
}

// x -> q, scale
PyObject* quantize_rows(PyObject* const* o) {
  Call c{"quantize_rows"};
  lipz_quantize_rows_args a{};
  a.struct_size = sizeof a;
  a.x = c.first(o[0], "x", WIDE);
  a.groups = c.groups, a.rows = c.rows, a.dim = c.cols;
  Tensor q, scale;
  a.q = c.fresh(q, c.rows, c.cols, E4M3);
  a.scale = c.fresh(scale, c.rows);
  run(c, lipz_quantize_rows, a);
  return results(give(q), give(scale));
}

// x, w, bias, act's code, slope, residual, x_scale, w_scale, out_dtype, keep, out -> y, pre
PyObject* linear(PyObject* const* o) {
  Call c{"linear"};
  lipz_linear_checkpoint_args kept{};
  lipz_linear_args& a = kept.call;
  kept.struct_size = sizeof kept;
  a.struct_size = sizeof a;
  a.x = c.first(o[0], "x", bit(LIPZ_BF16) | bit(LIPZ_E4M3));
  const Tensor& w = c.tensor(o[1], "w");
  if (w.dim() != (c.grouped ? 3 : 2)) c.refuse("w must be a CUDA tensor with x's number of dimensions");
  const int64_t n = w.size(-2);
  a.groups = c.groups, a.rows = c.rows, a.k = c.cols, a.n = n;
  a.w = c.mat(o[1], "w", n, c.cols, bit(a.x.type));
  a.bias = c.vec(o[2], "bias", n);
  a.act = (int)PyLong_AsLong(o[3]);
  a.slope = number(o[4]);
  const ScalarType type = c.result_type(o[8], "out_dtype");
  const bool own = o[10] != Py_None;
  if (own) a.y = c.target(o[10], "out", c.rows, n, bit(type_of(type)));
  a.residual = c.mat(o[5], "residual", c.rows, n, bit(type_of(type)));
  const bool bytes = a.x.type == LIPZ_E4M3;
  if ((o[6] != Py_None) != bytes || (o[7] != Py_None) != bytes)
    c.refuse("x_scale and w_scale go with 8-bit operands, and with them alone");
  a.x_scale = c.vec(o[6], "x_scale", c.rows);
  a.w_scale = c.vec(o[7], "w_scale", n);
  const int keep = keep_of(c, o[9]);
  Tensor y, pre, blocks;
  if (!own) a.y = c.fresh(y, c.rows, n, type);
  if (keep == 1) a.pre = c.fresh(pre, c.rows, n, BF16);
  if (keep == 2) {
    kept.pre = c.fresh(pre, blocks, c.rows, n);
    run(c, lipz_linear_checkpoint_workspace, lipz_linear_checkpoint, kept, a);
  } else {
    run(c, lipz_linear_workspace, lipz_linear, a);
  }
  if (own) c.wrote(o[10]);
  return results(own ? given(o[10]) : give(y), keep == 2 ? give(pre, blocks) : give(pre));
}

// dy, x, w, act's code, slope, pre, want_dx, want_dw, want_db, dx_dtype, dw_dtype -> dx, dw, db
PyObject* linear_backward(PyObject* const* o) {
  Call c{"linear_backward"};
  lipz_linear_backward_checkpoint_args kept{};
  lipz_linear_backward_args& a = kept.call;
  kept.struct_size = sizeof kept;
  a.struct_size = sizeof a;
  a.dy = c.first(o[0], "dy", HALF);
  const bool x_kept = c.is_checkpoint(o[1]);
  const Tensor& x = c.tensor(x_kept ? PyTuple_GET_ITEM(o[1], 0) : o[1], "x");
  if (x.dim() != (c.grouped ? 3 : 2)) c.refuse("x must be a CUDA tensor with dy's number of dimensions");
  c.require(o[2], "w");
  const int64_t n = c.cols, k = x.size(-1);
  a.groups = c.groups, a.rows = c.rows, a.k = k, a.n = n;
  if (x_kept) kept.x = c.blocks(o[1], "x", c.rows, k);
  else a.x = c.mat(o[1], "x", c.rows, k, HALF);
  a.w = c.mat(o[2], "w", n, k, HALF);
  a.act = (int)PyLong_AsLong(o[3]);
  a.slope = number(o[4]);
  if (a.act != LIPZ_ACT_NONE) {
    if (o[5] == Py_None) c.refuse("an activation needs pre");
    if (c.is_checkpoint(o[5])) kept.pre = c.blocks(o[5], "pre", c.rows, n);
    else a.pre = c.mat(o[5], "pre", c.rows, n, HALF);
  }
  const ScalarType dx_type = c.result_type(o[9], "dx_dtype"), dw_type = c.result_type(o[10], "dw_dtype");
  Tensor dx, dw, db;
  if (truth(o[6])) a.dx = c.fresh(dx, c.rows, k, dx_type);
  if (truth(o[7])) a.dw = c.fresh(dw, n, k, dw_type);
  if (truth(o[8])) a.db = c.fresh(db, n);
  if (kept.x.data || kept.pre.data)
    run(c, lipz_linear_backward_checkpoint_workspace, lipz_linear_backward_checkpoint, kept, a);
  else
    run(c, lipz_linear_backward_workspace, lipz_linear_backward, a);
  return results(give(dx), give(dw), give(db));
}

void raise(const Refusal& r) {
  PyObject* e = PyObject_CallFunction(g_error, "is", r.code, r.what.c_str());
  if (!e) return;
  PyErr_SetObject((PyObject*)Py_TYPE(e), e);
  Py_DECREF(e);
}

// A call of N positional arguments; refusals and torch's errors become Python's.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* o, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected", N);
    return nullptr;
  }
  try {
    return F(o);
  } catch (const Refusal& r) {
    raise(r);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define ENTRY(f, n) {#f, (PyCFunction)(void (*)())entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(rmsnorm, 7), ENTRY(rmsnorm_backward, 6), ENTRY(quantize_rows, 1),
                         ENTRY(linear, 11), ENTRY(linear_backward, 11), ENTRY(layernorm, 8),
                         ENTRY(layernorm_backward, 8), ENTRY(checkpoint_rows, 1), ENTRY(restore_rows, 4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "torch_operators", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_torch_operators() {
  PyObject* m = PyModule_Create(&module);
  PyObject* package = m ? PyImport_ImportModule("paper_1811_12843_gb300") : nullptr;
  g_error = package ? PyObject_GetAttrString(package, "LipzError") : nullptr;
  Py_XDECREF(package);
  // the sizes of the argument structures that this was compiled with
  PyObject* sizes = g_error ? Py_BuildValue("nnnnnnnnnnn", sizeof(lipz_rmsnorm_args),
                                            sizeof(lipz_rmsnorm_backward_args), sizeof(lipz_quantize_rows_args),
                                            sizeof(lipz_linear_args), sizeof(lipz_linear_backward_args),
                                            sizeof(lipz_layernorm_args), sizeof(lipz_layernorm_backward_args),
                                            sizeof(lipz_checkpoint_rows_args), sizeof(lipz_restore_rows_args),
                                            sizeof(lipz_linear_checkpoint_args),
                                            sizeof(lipz_linear_backward_checkpoint_args))
                            : nullptr;
  if (!sizes || PyModule_AddObject(m, "SIZES", sizes) < 0) {
    Py_XDECREF(m);
    return nullptr;
  }
  return m;
}
