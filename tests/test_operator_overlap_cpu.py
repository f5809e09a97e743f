"""Outputs that share memory with other arguments are refused, without a GPU: the comparison of two strided
regions against the bytes themselves, and the calls' refusals."""

import ctypes

import pytest

from helpers import native_program, run_program

PROGRAM = r"""
#include "operators.cu"
#include <random>
#include <set>

static std::set<uintptr_t> bytes(const Region& r) {
  std::set<uintptr_t> s;
  for (int64_t g = 0; g < r.groups; ++g)
    for (int64_t i = 0; i < r.rows; ++i)
      for (int64_t b = 0; b < r.width; ++b) s.insert(r.at + g * r.group + i * r.row + b);
  return s;
}

int main() {
  std::mt19937 rng(5);
  auto any = [&](int lo, int hi) { return (int64_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
  int together = 0, apart = 0, unknown = 0;
  for (int n = 0; n < 60000; ++n) {
    const int64_t row = any(0, 40), group = any(0, 1) ? any(0, 12) : any(20, 90);
    Region r[2];
    for (Region& q : r) {
      const bool own = n % 4 == 0;  // strides of its own
      q = Region::of((void*)(uintptr_t)any(1000, 1150), any(1, 9), any(0, 5), own ? any(0, 20) : row, any(0, 3),
                     own ? any(0, 60) : group);
      if (n % 5 == 0) q = q.joined();
    }
    const std::set<uintptr_t> a = bytes(r[0]), b = bytes(r[1]);
    bool shared = false;
    for (uintptr_t x : a) shared = shared || b.count(x);
    const Region p = r[0].joined(), q = r[1].joined();
    const bool exact =
        (p.rows < 2 || q.rows < 2 || p.row == q.row) && (p.groups < 2 || q.groups < 2 || p.group == q.group);
    if (meet(r[0], r[1]) != meet(r[1], r[0]) || (meet(r[0], r[1]) ? !shared : exact && shared)) {
      for (const Region& x : r)
        printf("%d %d x %d rows %d apart, %d groups %d apart\n", (int)x.at, (int)x.width, (int)x.rows, (int)x.row,
               (int)x.groups, (int)x.group);
      return 1;
    }
    if (meet(r[0], r[0]) != (r[0].width && r[0].rows && r[0].groups)) return 2;
    ++(meet(r[0], r[1]) ? together : shared ? unknown : apart);
  }
  printf("%d together, %d apart, %d unknown\n", together, apart, unknown);
  return together < 5000 || apart < 5000;
}
"""


def test_regions_against_their_bytes(tmp_path_factory):
    run_program(native_program(tmp_path_factory, "operator_overlap", PROGRAM, replaces=("operators.cu",)))


@pytest.fixture(scope="module")
def L():
    from paper_1811_12843_gb300 import _build
    _build.build()
    import paper_1811_12843_gb300 as lib
    lib.load()
    return lib


def _args(kind, **kw):
    a = kind()
    a.struct_size = ctypes.sizeof(a)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_calls_refuse_outputs_over_other_arguments(L):
    """(Every call here is refused: the addresses are no memory.)"""
    MB = 1 << 20
    B, F, Q = L.LIPZ_BF16, L.LIPZ_FP32, L.LIPZ_E4M3

    def mat(at, row=64, type=B, group=0):
        return L.lipz_mat(at, group, row, type, 0)

    def vec(at, group=0):
        return L.lipz_vec(at, group)

    def norm(**kw):
        a = dict(groups=1, rows=40, dim=64, eps=1e-6, x=mat(MB), residual=mat(2 * MB), sum=mat(3 * MB), y=mat(4 * MB),
                 weight=vec(5 * MB), rstd=vec(6 * MB))
        return L.lipz_rmsnorm, _args(L.lipz_rmsnorm_args, **dict(a, **kw))

    def back(**kw):
        a = dict(groups=1, rows=40, dim=64, dy=mat(MB), s=mat(2 * MB), dsum=mat(3 * MB), dx=mat(4 * MB),
                 weight=vec(5 * MB), rstd=vec(6 * MB), dweight=vec(7 * MB), workspace=16 * MB, workspace_bytes=16 * MB)
        return L.lipz_rmsnorm_backward, _args(L.lipz_rmsnorm_backward_args, **dict(a, **kw))

    def quant(**kw):
        a = dict(groups=1, rows=40, dim=64, x=mat(MB), q=mat(2 * MB, 64, Q), scale=vec(3 * MB))
        return L.lipz_quantize_rows, _args(L.lipz_quantize_rows_args, **dict(a, **kw))

    def linear(**kw):
        a = dict(groups=1, rows=40, k=64, n=64, x=mat(MB), w=mat(2 * MB), residual=mat(3 * MB), y=mat(4 * MB),
                 bias=vec(5 * MB), workspace=16 * MB, workspace_bytes=16 * MB)
        return L.lipz_linear, _args(L.lipz_linear_args, **dict(a, **kw))

    def linear_back(**kw):
        a = dict(groups=1, rows=40, k=64, n=64, dy=mat(MB), x=mat(2 * MB), w=mat(3 * MB), dx=mat(4 * MB),
                 dw=mat(5 * MB), db=vec(6 * MB), workspace=16 * MB, workspace_bytes=16 * MB)
        return L.lipz_linear_backward, _args(L.lipz_linear_backward_args, **dict(a, **kw))

    end = 39 * 128 + 126  # the last element of a matrix
    cases = [
        (linear(y=mat(MB)), "y overlaps x"), (linear(y=mat(MB - end)), "y overlaps x"),
        (linear(y=mat(MB + end)), "y overlaps x"), (linear(y=mat(2 * MB + 64)), "y overlaps w"),
        (linear(y=mat(3 * MB + 128)), "y overlaps residual"), (linear(y=mat(3 * MB, 96)), "y overlaps residual"),
        (linear(y=mat(MB + 192, 256), x=mat(MB, 256), k=100), "y overlaps x"),
        (linear(y=mat(5 * MB, type=F), residual=mat(3 * MB, type=F)), "y overlaps bias"),
        (linear(pre=mat(4 * MB)), "pre overlaps y"), (linear(pre=mat(3 * MB)), "pre overlaps residual"),
        (linear(x=mat(MB, type=Q), w=mat(2 * MB, type=Q), x_scale=vec(7 * MB), w_scale=vec(4 * MB + 64)),
         "y overlaps w_scale"),
        (linear(groups=3, y=mat(MB, group=64 * 64), x=mat(MB, 256), residual=mat(None)), "y overlaps x"),
        (norm(sum=mat(MB + 128)), "sum overlaps x"), (norm(y=mat(MB, type=Q), scale=vec(8 * MB)), "y overlaps x"),
        (norm(y=mat(3 * MB)), "y overlaps sum"), (norm(sum=mat(MB), y=mat(MB)), "y overlaps sum"),
        (norm(y=mat(5 * MB)), "y overlaps weight"), (norm(rstd=vec(4 * MB + 8)), "rstd overlaps y"),
        (back(dx=mat(2 * MB + 64)), "dx overlaps s"), (back(dweight=vec(3 * MB)), "dweight overlaps dsum"),
        (back(dx=mat(6 * MB)), "dx overlaps rstd"), (back(dweight=vec(5 * MB)), "dweight overlaps weight"),
        (quant(q=mat(MB, 64, Q)), "q overlaps x"), (quant(scale=vec(MB + 4)), "scale overlaps x"),
        (quant(q=mat(MB, 128, Q), x=mat(MB, 64, F)), "q overlaps x"),
        (linear_back(dx=mat(MB)), "dx overlaps dy"), (linear_back(dw=mat(3 * MB)), "dw overlaps w"),
        (linear_back(dw=mat(4 * MB + 2)), "dw overlaps dx"), (linear_back(db=vec(2 * MB)), "db overlaps x"),
    ]
    for (call, args), what in cases:
        with pytest.raises(L.LipzError) as e:
            call(args)
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), (what, str(e.value))
