"""The layer norm's and the checkpoints' calls without a GPU: argument structures, and refusals before any launch."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

MB = 1 << 20


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


def _mat(L, type, row, group=0, data=MB):
    return L.lipz_mat(data, group, row, type, 0)


def _blocks(L, cols, data, scale, rows=4, **kw):
    b = L.lipz_blocks(data, rows * cols, cols, scale, rows * -(-cols // 16), -(-cols // 16))
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _norm(L, **kw):
    a = dict(groups=1, rows=4, dim=64, eps=1e-5, x=_mat(L, L.LIPZ_BF16, 64, 256, MB),
             y=_mat(L, L.LIPZ_BF16, 64, 256, 2 * MB), weight=L.lipz_vec(3 * MB, 64))
    return _args(L.lipz_layernorm_args, **{**a, **kw})


def _back(L, **kw):
    a = dict(groups=1, rows=4, dim=64, dy=_mat(L, L.LIPZ_BF16, 64, 256, MB), s=_mat(L, L.LIPZ_BF16, 64, 256, 2 * MB),
             dx=_mat(L, L.LIPZ_BF16, 64, 256, 3 * MB), weight=L.lipz_vec(4 * MB, 64), mean=L.lipz_vec(5 * MB, 4),
             rstd=L.lipz_vec(6 * MB, 4))
    return _args(L.lipz_layernorm_backward_args, **{**a, **kw})


def _linear(L, kept, **kw):
    a = dict(groups=1, rows=4, k=64, n=32, x=_mat(L, 1, 64, 256, MB), w=_mat(L, 1, 64, 2048, 2 * MB),
             y=_mat(L, 1, 32, 128, 3 * MB))
    return _args(L.lipz_linear_checkpoint_args, call=_args(L.lipz_linear_args, **{**a, **kw}), pre=kept)


def _linear_back(L, kept_x=None, kept_pre=None, **kw):
    a = dict(groups=1, rows=4, k=64, n=32, act=L.LIPZ_ACT_GELU, dy=_mat(L, 1, 32, 128, MB),
             w=_mat(L, 1, 64, 2048, 2 * MB), dx=_mat(L, 1, 64, 256, 3 * MB), dw=_mat(L, 1, 64, 2048, 4 * MB))
    call = _args(L.lipz_linear_backward_args, **{**a, **kw})
    return _args(L.lipz_linear_backward_checkpoint_args, call=call, x=kept_x or L.lipz_blocks(),
                 pre=kept_pre or L.lipz_blocks())


def test_packed_arguments_have_the_structures_sizes(L):
    from paper_1811_12843_gb300 import operators as ops
    for struct, packed in ((L.lipz_layernorm_args, ops._S_LAYERNORM),
                           (L.lipz_layernorm_backward_args, ops._S_LAYERNORM_BACKWARD),
                           (L.lipz_checkpoint_rows_args, ops._S_CHECKPOINT),
                           (L.lipz_restore_rows_args, ops._S_RESTORE),
                           (L.lipz_linear_checkpoint_args, ops._S_LINEAR_CHECKPOINT),
                           (L.lipz_linear_backward_checkpoint_args, ops._S_LINEAR_BACKWARD_CHECKPOINT)):
        assert ctypes.sizeof(struct) == packed.size
    assert (ops._load().SIZES == tuple(s.size for s in ops._STRUCTURES))


def test_bad_arguments_are_refused(L):
    """Addresses here are no memory at all: a call that launched anything would fail otherwise."""
    B, F, Q = L.LIPZ_BF16, L.LIPZ_FP32, L.LIPZ_E4M3
    c = _blocks(L, 64, 8 * MB, 9 * MB)
    wide = _blocks(L, 32, 8 * MB, 9 * MB)

    def rows(**kw):
        a = dict(groups=1, rows=4, dim=64, x=_mat(L, B, 64), c=c)
        return _args(L.lipz_checkpoint_rows_args, **{**a, **kw})

    def back(**kw):
        a = dict(groups=1, rows=4, dim=64, act=0, y=_mat(L, B, 64), c=c)
        return _args(L.lipz_restore_rows_args, **{**a, **kw})

    cases = [
        (L.lipz_layernorm, _norm(L, struct_size=8), "struct_size"),
        (L.lipz_layernorm, _norm(L, dim=0), "dim"), (L.lipz_layernorm, _norm(L, dim=16385), "dim"),
        (L.lipz_layernorm, _norm(L, eps=-1.0), "eps"), (L.lipz_layernorm, _norm(L, eps=float("nan")), "eps"),
        (L.lipz_layernorm, _norm(L, weight=L.lipz_vec(None, 0)), "weight is null"),
        (L.lipz_layernorm, _norm(L, bias=L.lipz_vec(MB + 2, 0)), "bias is not aligned"),
        (L.lipz_layernorm, _norm(L, y=_mat(L, F, 64, 0, 2 * MB)), "y has a type"),
        (L.lipz_layernorm, _norm(L, y=_mat(L, Q, 64, 0, 2 * MB)), "scale is null"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, None, 9 * MB)), "kept is null"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, 8 * MB, None)), "kept's scale is null"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, 8 * MB, 9 * MB, row=63)), "kept has a row stride"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, 8 * MB, 9 * MB, scale_row=3)), "kept's scale has a row"),
        (L.lipz_layernorm, _norm(L, kept=c, residual=_mat(L, B, 64, 0, 10 * MB)), "kept needs sum"),
        (L.lipz_layernorm, _norm(L, groups=2, kept=_blocks(L, 64, 8 * MB, 9 * MB, group=100)), "kept has groups"),
        (L.lipz_layernorm_backward, _back(L, s=_mat(L, F, 64, 0, 2 * MB)), "s has a type"),
        (L.lipz_layernorm_backward, _back(L, s=_mat(L, B, 64, 0, None)), "s is null"),
        (L.lipz_layernorm_backward, _back(L, kept=c), "s is given twice"),
        (L.lipz_layernorm_backward, _back(L, s=L.lipz_mat(), kept=_blocks(L, 64, 8 * MB, None)), "scale is null"),
        (L.lipz_layernorm_backward, _back(L, mean=L.lipz_vec(None, 0)), "mean is null"),
        (L.lipz_layernorm_backward, _back(L, rstd=L.lipz_vec(None, 0)), "rstd is null"),
        (L.lipz_layernorm_backward, _back(L, dx=_mat(L, B, 63, 0, 3 * MB)), "dx has a row stride"),
        (L.lipz_checkpoint_rows, rows(dim=0), "dim"), (L.lipz_checkpoint_rows, rows(x=_mat(L, Q, 64)), "x has a type"),
        (L.lipz_checkpoint_rows, rows(c=L.lipz_blocks()), "c is null"),
        (L.lipz_checkpoint_rows, rows(c=_blocks(L, 64, MB + 100, 9 * MB)), "c overlaps x"),
        (L.lipz_checkpoint_rows, rows(c=_blocks(L, 64, 8 * MB, 8 * MB + 255)), "overlaps c"),
        (L.lipz_restore_rows, back(act=6), "act"), (L.lipz_restore_rows, back(y=_mat(L, Q, 64)), "y has a type"),
        (L.lipz_restore_rows, back(c=_blocks(L, 64, MB + 1, 9 * MB)), "y overlaps c"),
        (L.lipz_restore_rows, back(c=_blocks(L, 64, 8 * MB, MB + 511)), "y overlaps c"),
        (L.lipz_linear_checkpoint, _linear(L, L.lipz_blocks()), "pre is null"),
        (L.lipz_linear_checkpoint, _linear(L, wide, pre=_mat(L, B, 32, 0, 7 * MB)), "pre is given twice"),
        (L.lipz_linear_checkpoint, _linear(L, wide, x=_mat(L, F, 64)), "x has a type"),
        (L.lipz_linear_checkpoint, _linear(L, wide, struct_size=8), "struct_size"),
        (L.lipz_linear_checkpoint, _linear(L, _blocks(L, 32, 3 * MB + 8, 9 * MB)), "pre overlaps y"),
        (L.lipz_linear_checkpoint, _linear(L, _blocks(L, 32, 8 * MB, 2 * MB)), "overlaps w"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, c, wide, x=_mat(L, B, 64, 0, 7 * MB)), "x is given twice"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, c, wide, pre=_mat(L, B, 32, 0, 7 * MB)), "pre is given"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, None, wide), "x is null"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, c, None), "pre is null"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, _blocks(L, 64, 8 * MB, None), wide), "x's scale is null"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, c, wide, dx=_mat(L, B, 64, 0, 8 * MB)), "dx overlaps"),
        (L.lipz_linear_backward_checkpoint, _linear_back(L, c, wide, dw=_mat(L, B, 64, 0, 9 * MB - 4000)),
         "dw overlaps"),
    ]
    for call, args, what in cases:
        with pytest.raises(L.LipzError) as e:
            call(args)
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), (what, str(e.value))
        assert what in L.lipz_operator_error()


def test_outputs_over_other_arguments_are_refused(L):
    V, B = L.lipz_vec, L.LIPZ_BF16
    c = _blocks(L, 64, 8 * MB, 9 * MB)
    cases = [
        (L.lipz_layernorm, _norm(L, y=_mat(L, B, 64, 0, MB + 128)), "y overlaps x"),
        (L.lipz_layernorm, _norm(L, mean=V(MB + 16, 4)), "mean overlaps x"),
        (L.lipz_layernorm, _norm(L, mean=V(10 * MB, 4), rstd=V(10 * MB + 8, 4)), "rstd overlaps mean"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, 2 * MB + 8, 9 * MB)), "kept overlaps y"),
        (L.lipz_layernorm, _norm(L, kept=_blocks(L, 64, 8 * MB, 3 * MB)), "overlaps weight"),
        (L.lipz_layernorm, _norm(L, kept=c, mean=V(9 * MB + 12, 4)), "overlaps mean"),
        (L.lipz_layernorm_backward, _back(L, dx=_mat(L, B, 64, 0, 2 * MB + 2)), "dx overlaps s"),
        (L.lipz_layernorm_backward, _back(L, dweight=V(5 * MB, 64)), "dweight overlaps mean"),
        (L.lipz_layernorm_backward, _back(L, dweight=V(11 * MB, 64), dbias=V(11 * MB + 128, 64)), "dbias overlaps"),
        (L.lipz_layernorm_backward, _back(L, s=L.lipz_mat(), kept=c, dx=_mat(L, B, 64, 0, 8 * MB)), "dx overlaps"),
    ]
    for call, args, what in cases:
        with pytest.raises(L.LipzError) as e:
            call(args)
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), (what, str(e.value))


def test_workspace_that_is_missing_or_small_is_refused(L):
    cases = []
    back = _back(L, rows=1000, dweight=L.lipz_vec(64 * MB, 64), dy=_mat(L, 1, 64, 0, 65 * MB),
                 s=_mat(L, 1, 64, 0, 66 * MB), dx=_mat(L, 1, 64, 0, 67 * MB), rstd=L.lipz_vec(68 * MB, 0),
                 mean=L.lipz_vec(69 * MB, 0))
    cases.append((L.lipz_layernorm_backward_workspace, L.lipz_layernorm_backward, back, back))
    x, pre = _blocks(L, 64, 8 * MB, 9 * MB, rows=100), _blocks(L, 32, 10 * MB, 11 * MB, rows=100)
    lin = _linear_back(L, x, pre, rows=100, db=L.lipz_vec(12 * MB, 0))
    cases.append((L.lipz_linear_backward_checkpoint_workspace, L.lipz_linear_backward_checkpoint, lin, lin.call))
    for query, call, a, where in cases:
        need = query(a)
        assert need > 0
        for data, size in ((None, need), (256, need - 1), (128, need)):
            where.workspace, where.workspace_bytes = data, size
            with pytest.raises(L.LipzError) as e:
                call(a)
            assert e.value.code == L.LIPZ_ERR_INVALID and "workspace" in str(e.value)


def test_nothing_to_do(L):
    """No rows or no groups: nothing is launched, and nothing but the sums over no rows is written."""
    none = L.lipz_mat()
    assert L.lipz_layernorm(_norm(L, rows=0, x=none, y=none)) == L.LIPZ_OK
    assert L.lipz_layernorm(_norm(L, groups=0, x=none, y=none)) == L.LIPZ_OK
    assert L.lipz_layernorm_backward(_back(L, groups=0)) == L.LIPZ_OK
    assert L.lipz_checkpoint_rows(_args(L.lipz_checkpoint_rows_args, groups=1, rows=0, dim=8)) == L.LIPZ_OK
    assert L.lipz_restore_rows(_args(L.lipz_restore_rows_args, groups=1, rows=0, dim=8)) == L.LIPZ_OK


def test_tensors_that_are_not_on_a_gpu_are_refused(L):
    from paper_1811_12843_gb300 import operators as ops
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    c = ops.Checkpoint(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 4, dtype=torch.uint8))
    for f in (lambda: ops.layernorm(x, torch.ones(64)), lambda: ops.checkpoint_rows(x), lambda: ops.restore_rows(c),
              lambda: ops.linear(x, w, keep="int8"), lambda: ops.linear_backward(torch.zeros(4, 8), c, w),
              lambda: ops.layernorm_backward(x, c, torch.ones(4), torch.ones(4), torch.ones(64))):
        with pytest.raises(L.LipzError) as e:
            f()
        assert e.value.code == L.LIPZ_ERR_INVALID and "CUDA" in str(e.value)
