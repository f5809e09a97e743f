"""The residual-block operators without a GPU: argument structures, and refusals before any launch."""

import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    from paper_1811_12843_gb300 import _build
    _build.build()
    import paper_1811_12843_gb300 as lib
    lib.load()
    return lib


def _mat(L, type, row, group=0, data=256):
    return L.lipz_mat(data, group, row, type, 0)


def _linear(L, **kw):
    a = L.lipz_linear_args()
    a.struct_size = ctypes.sizeof(a)
    a.groups, a.rows, a.k, a.n = 1, 4, 64, 32
    a.x, a.w, a.y = (_mat(L, L.LIPZ_BF16, 64), _mat(L, L.LIPZ_BF16, 64), _mat(L, L.LIPZ_BF16, 32))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _norm(L, **kw):
    a = L.lipz_rmsnorm_args()
    a.struct_size = ctypes.sizeof(a)
    a.groups, a.rows, a.dim, a.eps = 1, 4, 64, 1e-6
    a.x, a.y = _mat(L, L.LIPZ_BF16, 64), _mat(L, L.LIPZ_BF16, 64)
    a.weight = L.lipz_vec(256, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_packed_arguments_have_the_structures_sizes(L):
    from paper_1811_12843_gb300 import operators as ops
    for struct, packed in ((L.lipz_rmsnorm_args, ops._S_RMSNORM),
                           (L.lipz_rmsnorm_backward_args, ops._S_RMSNORM_BACKWARD),
                           (L.lipz_quantize_rows_args, ops._S_QUANTIZE),
                           (L.lipz_linear_args, ops._S_LINEAR),
                           (L.lipz_linear_backward_args, ops._S_LINEAR_BACKWARD)):
        assert ctypes.sizeof(struct) == packed.size


def test_bad_arguments_are_refused(L):
    """Addresses here are no memory at all: a call that launched anything would fail otherwise."""
    B, F, Q = L.LIPZ_BF16, L.LIPZ_FP32, L.LIPZ_E4M3
    cases = [
        (L.lipz_linear, _linear(L, struct_size=8), "struct_size"),
        (L.lipz_linear, _linear(L, k=0), "k must"), (L.lipz_linear, _linear(L, n=0), "n must"),
        (L.lipz_linear, _linear(L, rows=-1), "rows"), (L.lipz_linear, _linear(L, groups=70000), "groups"),
        (L.lipz_linear, _linear(L, act=6), "act"), (L.lipz_linear, _linear(L, act=-1), "act"),
        (L.lipz_linear, _linear(L, x=_mat(L, F, 64)), "x has a type"),
        (L.lipz_linear, _linear(L, w=_mat(L, Q, 64)), "w has a type"),
        (L.lipz_linear, _linear(L, y=_mat(L, Q, 32)), "y has a type"),
        (L.lipz_linear, _linear(L, y=_mat(L, 7, 32)), "y has a type"),
        (L.lipz_linear, _linear(L, y=_mat(L, B, 31)), "y has a row stride"),
        (L.lipz_linear, _linear(L, y=_mat(L, B, 32, data=257)), "y is not aligned"),
        (L.lipz_linear, _linear(L, y=_mat(L, B, 32, data=None)), "y is null"),
        (L.lipz_linear, _linear(L, residual=_mat(L, F, 32)), "residual has a type"),
        (L.lipz_linear, _linear(L, pre=_mat(L, F, 32)), "pre has a type"),
        (L.lipz_linear, _linear(L, bias=L.lipz_vec(258, 0)), "bias is not aligned"),
        (L.lipz_linear, _linear(L, groups=2), "y has groups that overlap"),
        (L.lipz_linear, _linear(L, groups=2, y=_mat(L, B, 32, 127)), "y has groups that overlap"),
        (L.lipz_linear, _linear(L, groups=2, x=_mat(L, B, 64, -4)), "x has a negative"),
        (L.lipz_linear, _linear(L, x=_mat(L, Q, 64), w=_mat(L, Q, 64)), "x_scale is null"),
        (L.lipz_linear, _linear(L, groups=2 ** 15, rows=2 ** 17), "2^31"),
        (L.lipz_rmsnorm, _norm(L, dim=0), "dim"), (L.lipz_rmsnorm, _norm(L, dim=16385), "dim"),
        (L.lipz_rmsnorm, _norm(L, eps=-1.0), "eps"), (L.lipz_rmsnorm, _norm(L, eps=float("nan")), "eps"),
        (L.lipz_rmsnorm, _norm(L, weight=L.lipz_vec(None, 0)), "weight is null"),
        (L.lipz_rmsnorm, _norm(L, y=_mat(L, F, 64)), "y has a type"),
        (L.lipz_rmsnorm, _norm(L, y=_mat(L, Q, 64)), "scale is null"),
        (L.lipz_rmsnorm, _norm(L, sum=_mat(L, F, 64)), "sum has a type"),
    ]
    for call, args, what in cases:
        with pytest.raises(L.LipzError) as e:
            call(args)
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), str(e.value)
        assert what in L.lipz_operator_error()


def test_workspace_that_is_missing_or_small_is_refused(L):
    a = L.lipz_linear_backward_args()
    a.struct_size = ctypes.sizeof(a)
    a.groups, a.rows, a.k, a.n = 1, 100, 64, 32
    a.dy, a.x, a.w = _mat(L, 1, 32), _mat(L, 1, 64), _mat(L, 1, 64)
    a.pre, a.dx, a.dw = _mat(L, 1, 32), _mat(L, 1, 64), _mat(L, 1, 64)
    a.db, a.act = L.lipz_vec(256, 0), L.LIPZ_ACT_SILU
    need = L.lipz_linear_backward_workspace(a)
    assert need >= 100 * 32 * 2
    for data, size in ((None, need), (256, need - 1), (128, need)):
        a.workspace, a.workspace_bytes = data, size
        with pytest.raises(L.LipzError) as e:
            L.lipz_linear_backward(a)
        assert e.value.code == L.LIPZ_ERR_INVALID and "workspace" in str(e.value)


def test_tensors_that_are_not_on_a_gpu_are_refused(L):
    from paper_1811_12843_gb300 import operators as ops
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    for f in (lambda: ops.rmsnorm(x, torch.ones(64)), lambda: ops.quantize_rows(x),
              lambda: ops.linear(x, w), lambda: ops.linear_backward(torch.zeros(4, 8), x, w),
              lambda: ops.rmsnorm_backward(x, x, torch.ones(4), torch.ones(64))):
        with pytest.raises(L.LipzError) as e:
            f()
        assert e.value.code == L.LIPZ_ERR_INVALID and "CUDA" in str(e.value)


def test_status_without_a_failure(L):
    assert L.lipz_operator_status() == L.LIPZ_OK
