"""The operators of a pre-norm residual block on torch tensors (C ABI: include/lipz.h).

    h, s = rmsnorm(x + s)          a = act(h W1^T + b1)          s' = a W2^T + b2 + s

forward and backward in bf16, and forward over 8-bit operands, for one network or for a population
of them: tensors are [rows, columns], or [groups, rows, columns] with weights per group. Columns
must be adjacent; rows and groups may be strided, and a group stride of 0 (``expand``) shares an
input between the groups. An output may not overlap an input unless its call says so. Every call
runs the library's CUDA kernels on the current stream of the tensors' device, allocates its outputs
as torch does, waits for nothing, and may be captured in a CUDA graph. What the library does not
take raises ``LipzError`` with nothing launched. Nothing here records an autograd graph: the
backward passes are calls of their own.
"""

import ctypes
import struct
from typing import NamedTuple, Optional

import torch

from . import (LIPZ_BF16, LIPZ_E4M3, LIPZ_ERR_INVALID, LIPZ_FP32, LIPZ_OK, LipzError, load,
               lipz_operator_error)

__all__ = ["Norm", "rmsnorm", "rmsnorm_backward", "quantize_rows", "linear", "linear_backward",
           "ACTIVATIONS"]

ACTIVATIONS = {"none": 0, "relu": 1, "lrelu": 2, "tanh": 3, "gelu": 4, "silu": 5}

_F32, _BF16, _E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
_TYPE = {_F32: LIPZ_FP32, _BF16: LIPZ_BF16, _E4M3: LIPZ_E4M3}

# the argument structures of include/lipz.h
_MAT, _VEC = "QqqiI", "Qq"
_S_RMSNORM = struct.Struct("=If3q" + 4 * _MAT + 3 * _VEC)
_S_RMSNORM_BACKWARD = struct.Struct("=II3q" + 4 * _MAT + 3 * _VEC + "QQ")
_S_QUANTIZE = struct.Struct("=II3q" + 2 * _MAT + _VEC)
_S_LINEAR = struct.Struct("=IifI4q" + 5 * _MAT + 3 * _VEC + "QQ")
_S_LINEAR_BACKWARD = struct.Struct("=IifI4q" + 6 * _MAT + _VEC + "QQ")
_NO_MAT, _NO_VEC = (0, 0, 0, 0, 0), (0, 0)
_WIDE = (_BF16, _F32)


def _refuse(call, what):
    raise LipzError(LIPZ_ERR_INVALID, "%s: %s" % (call, what))


def _refuse_tensor(call, name, t, shape, dtypes, device):
    """Says why a tensor is refused."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _refuse(call, "%s must be a CUDA tensor on the same device as the others" % name)
    if t.dtype not in dtypes:
        _refuse(call, "%s has dtype %s, taken are %s" % (name, t.dtype, ", ".join(map(str, dtypes))))
    if t.shape != shape:
        _refuse(call, "%s has shape %s, not %s" % (name, list(t.shape), list(shape)))
    _refuse(call, "%s: columns must be adjacent" % name)


# (These run for every tensor of every call, next to kernels of a few microseconds.)
def _mat(call, name, t, shape, dtypes, device):
    """(address, group stride, row stride, type, 0) of a checked matrix."""
    if t is None:
        return _NO_MAT
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.shape == shape and t.get_device() == device:
        st = t.stride()
        if st[-1] == 1 or shape[-1] <= 1 or not t.numel():
            return t.data_ptr(), st[0] if len(st) == 3 else 0, st[-2], _TYPE[t.dtype], 0
    _refuse_tensor(call, name, t, shape, dtypes, device)


def _vec(call, name, t, shape, device):
    """(address, group stride) of a checked fp32 vector."""
    if t is None:
        return _NO_VEC
    if isinstance(t, torch.Tensor) and t.dtype is _F32 and t.shape == shape and t.get_device() == device:
        st = t.stride()
        if st[-1] == 1 or shape[-1] <= 1 or not t.numel():
            return t.data_ptr(), st[0] if len(st) == 2 else 0
    _refuse_tensor(call, name, t, shape, (_F32,), device)


def _first(call, name, t, dtypes):
    """(shape, groups, rows, columns, device index, matrix) of the tensor that a call's others go by."""
    if not isinstance(t, torch.Tensor) or t.get_device() < 0:
        _refuse(call, "%s must be a CUDA tensor" % name)
    s, st, dtype = t.shape, t.stride(), t.dtype
    if len(s) != 2 and len(s) != 3:
        _refuse(call, "%s must be [rows, columns] or [groups, rows, columns]" % name)
    if dtype not in dtypes or (st[-1] != 1 and s[-1] > 1 and t.numel()):
        _refuse_tensor(call, name, t, s, dtypes, t.get_device())
    if len(s) == 2:
        return s, 1, s[0], s[1], t.get_device(), (t.data_ptr(), 0, st[0], _TYPE[dtype], 0)
    return s, s[0], s[1], s[2], t.get_device(), (t.data_ptr(), st[0], st[1], _TYPE[dtype], 0)


def _act(call, act):
    code = ACTIVATIONS.get(act)
    if code is None:
        _refuse(call, "act must be one of %s (got %r)" % (", ".join(ACTIVATIONS), act))
    return code


# the handle of the device's current stream, and the current device, without the objects around them
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _raise(rc):
    raise LipzError(rc, lipz_operator_error())


def _run(name, args, device):
    """The library's call on the device's current stream."""
    if device != _current():
        with torch.cuda.device(device):
            return _run(name, args, device)
    rc = getattr(load(), name)(args, _stream(device))
    if rc:
        _raise(rc)


def _run_with_space(name, query, struct_, fields, dev, device):
    """The call with the workspace that it asks for."""
    if device != _current():
        with torch.cuda.device(device):
            return _run_with_space(name, query, struct_, fields, dev, device)
    lib, need, args = load(), ctypes.c_uint64(), struct_.pack(*fields, 0, 0)
    rc = getattr(lib, query)(args, ctypes.byref(need))
    if rc:
        _raise(rc)
    if need.value:
        work = torch.empty(need.value, dtype=torch.uint8, device=dev)
        args = struct_.pack(*fields, work.data_ptr(), need.value)
    rc = getattr(lib, name)(args, _stream(device))
    if rc:
        _raise(rc)


class Norm(NamedTuple):
    """rmsnorm's results; ``scale`` with 8 bits, ``rstd`` where it is kept, else None."""
    y: torch.Tensor
    sum: torch.Tensor
    scale: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]


def rmsnorm(x, weight, residual=None, eps=1e-6, e4m3=False, keep=False, sum_out=None) -> Norm:
    """s = x + residual, y = s weight / sqrt(mean(s^2) + eps) over the columns.

    x, residual: bf16 or fp32; weight [columns] (or [groups, columns]) fp32. ``sum`` is s in x's type
    (x itself without a residual), written to ``sum_out`` if given (it may be x or residual: the
    residual stream updated in place). y has x's type; with ``e4m3`` it is float8_e4m3fn and
    y scale[row] the values. ``keep``: return rstd, which the backward pass reads."""
    call = "rmsnorm"
    shape, groups, rows, dim, device, mx = _first(call, "x", x, _WIDE)
    dev, dtype = x.device, x.dtype
    dt = (dtype,)
    two = len(shape) == 2
    per_row, per_col = ((rows,), (dim,)) if two else ((groups, rows), (groups, dim))
    vw = _vec(call, "weight", weight, per_col, device)
    if weight is None:
        _refuse(call, "weight must be given")
    if residual is None:
        if sum_out is not None:
            _refuse(call, "sum_out needs a residual")
        total, mr, ms = x, _NO_MAT, _NO_MAT
    else:
        mr = _mat(call, "residual", residual, shape, dt, device)
        if sum_out is None:
            total = torch.empty(shape, dtype=dtype, device=dev)
            ms = (total.data_ptr(), rows * dim, dim, mx[3], 0)
        else:
            total, ms = sum_out, _mat(call, "sum_out", sum_out, shape, dt, device)
    y = torch.empty(shape, dtype=_E4M3 if e4m3 else dtype, device=dev)
    scale = torch.empty(per_row, dtype=_F32, device=dev) if e4m3 else None
    rstd = torch.empty(per_row, dtype=_F32, device=dev) if keep else None
    _run("lipz_rmsnorm", _S_RMSNORM.pack(
        _S_RMSNORM.size, eps, groups, rows, dim, *mx, *mr, *ms,
        y.data_ptr(), rows * dim, dim, LIPZ_E4M3 if e4m3 else mx[3], 0, *vw,
        scale.data_ptr() if e4m3 else 0, rows, rstd.data_ptr() if keep else 0, rows), device)
    return Norm(y, total, scale, rstd)


def rmsnorm_backward(dy, s, rstd, weight, dsum=None, want_dweight=True):
    """(dx, dweight) of rmsnorm: from its ``sum`` and ``rstd``, y's gradient, and dsum, the gradient
    that reaches the sum from elsewhere. dx is the gradient of x and of residual; dweight is fp32."""
    call = "rmsnorm_backward"
    shape, groups, rows, dim, device, ms = _first(call, "s", s, _WIDE)
    dev, dt = s.device, (s.dtype,)
    per_row, per_col = ((rows,), (dim,)) if len(shape) == 2 else ((groups, rows), (groups, dim))
    if dy is None or weight is None or rstd is None:
        _refuse(call, "dy, rstd and weight must be given")
    mats = _mat(call, "dy", dy, shape, dt, device) + ms + _mat(call, "dsum", dsum, shape, dt, device)
    vecs = _vec(call, "weight", weight, per_col, device) + _vec(call, "rstd", rstd, per_row, device)
    dx = torch.empty(shape, dtype=s.dtype, device=dev)
    dweight = torch.empty(per_col, dtype=_F32, device=dev) if want_dweight else None
    _run_with_space("lipz_rmsnorm_backward", "lipz_rmsnorm_backward_workspace", _S_RMSNORM_BACKWARD,
                    (_S_RMSNORM_BACKWARD.size, 0, groups, rows, dim, *mats, dx.data_ptr(), rows * dim,
                     dim, ms[3], 0, *vecs, dweight.data_ptr() if want_dweight else 0, dim),
                    dev, device)
    return dx, dweight


def quantize_rows(x):
    """(q, scale): x [.., rows, columns] (bf16 or fp32) in float8_e4m3fn with an fp32 scale per row,
    q scale the values."""
    call = "quantize_rows"
    shape, groups, rows, dim, device, mx = _first(call, "x", x, _WIDE)
    dev = x.device
    q = torch.empty(shape, dtype=_E4M3, device=dev)
    scale = torch.empty((rows,) if len(shape) == 2 else (groups, rows), dtype=_F32, device=dev)
    _run("lipz_quantize_rows",
         _S_QUANTIZE.pack(_S_QUANTIZE.size, 0, groups, rows, dim, *mx, q.data_ptr(), rows * dim, dim,
                          LIPZ_E4M3, 0, scale.data_ptr(), rows), device)
    return q, scale


def linear(x, w, bias=None, act="none", slope=0.2, residual=None, x_scale=None, w_scale=None,
           out_dtype=torch.bfloat16, keep=False, out=None):
    """(y, pre): u = x w^T (x_scale[row] w_scale[column]) + bias, y = act(u) + residual.

    x [.., rows, k] and w [.., n, k]: bf16, or float8_e4m3fn with both scales; bias fp32; residual and
    y: out_dtype (bf16 or fp32). y is written to ``out`` if given (it may be the residual). ``keep``:
    pre is u in bf16, which the backward pass reads (else None)."""
    call = "linear"
    x_shape, groups, rows, k, device, mx = _first(call, "x", x, (_BF16, _E4M3))
    dev = x.device
    if not isinstance(w, torch.Tensor) or w.dim() != len(x_shape):
        _refuse(call, "w must be a CUDA tensor with x's number of dimensions")
    n, code = w.shape[-2], _act(call, act)
    if len(x_shape) == 2:
        shape, w_shape, per_row, per_col = (rows, n), (n, k), (rows,), (n,)
    else:
        shape, w_shape, per_row, per_col = (groups, rows, n), (groups, n, k), (groups, rows), (groups, n)
    mw = _mat(call, "w", w, w_shape, (x.dtype,), device)
    if out_dtype is not _BF16 and out_dtype is not _F32:
        _refuse(call, "out_dtype must be bfloat16 or float32")
    if (x_scale is None) != (mx[3] != LIPZ_E4M3) or (w_scale is None) != (mx[3] != LIPZ_E4M3):
        _refuse(call, "x_scale and w_scale go with 8-bit operands, and with them alone")
    mr = _mat(call, "residual", residual, shape, (out_dtype,), device)
    vecs = (_vec(call, "x_scale", x_scale, per_row, device)
            + _vec(call, "w_scale", w_scale, per_col, device)
            + _vec(call, "bias", bias, per_col, device))
    if out is None:
        y = torch.empty(shape, dtype=out_dtype, device=dev)
        my = (y.data_ptr(), rows * n, n, _TYPE[out_dtype], 0)
    else:
        y, my = out, _mat(call, "out", out, shape, (out_dtype,), device)
    pre = torch.empty(shape, dtype=_BF16, device=dev) if keep else None
    mp = (pre.data_ptr(), rows * n, n, LIPZ_BF16, 0) if keep else _NO_MAT
    _run_with_space("lipz_linear", "lipz_linear_workspace", _S_LINEAR,
                    (_S_LINEAR.size, code, slope, 0, groups, rows, k, n, *mx, *mw, *mr, *my, *mp, *vecs),
                    dev, device)
    return y, pre


def linear_backward(dy, x, w, act="none", slope=0.2, pre=None, want_dx=True, want_dw=True,
                    want_db=True, dx_dtype=torch.bfloat16, dw_dtype=torch.bfloat16):
    """(dx, dw, db) of linear over bf16 operands: du = dy act'(pre), dx = du w, dw = du^T x, db the
    sums of du over the rows (fp32); None for what is not wanted. dx and dw: bf16 or fp32. The
    residual's gradient is dy."""
    call = "linear_backward"
    bf = (_BF16,)
    shape, groups, rows, n, device, mdy = _first(call, "dy", dy, bf)
    dev = dy.device
    if not isinstance(x, torch.Tensor) or x.dim() != len(shape):
        _refuse(call, "x must be a CUDA tensor with dy's number of dimensions")
    if w is None:
        _refuse(call, "w must be given")
    k, code = x.shape[-1], _act(call, act)
    if len(shape) == 2:
        x_shape, w_shape, per_col = (rows, k), (n, k), (n,)
    else:
        x_shape, w_shape, per_col = (groups, rows, k), (groups, n, k), (groups, n)
    if code and pre is None:
        _refuse(call, "act %r needs pre" % act)
    if dx_dtype not in _WIDE or dw_dtype not in _WIDE:
        _refuse(call, "dx_dtype and dw_dtype must be bfloat16 or float32")
    mats = (mdy + _mat(call, "x", x, x_shape, bf, device) + _mat(call, "w", w, w_shape, bf, device)
            + _mat(call, "pre", pre if code else None, shape, bf, device))
    dx = torch.empty(x_shape, dtype=dx_dtype, device=dev) if want_dx else None
    dw = torch.empty(w_shape, dtype=dw_dtype, device=dev) if want_dw else None
    db = torch.empty(per_col, dtype=_F32, device=dev) if want_db else None
    mx = (dx.data_ptr(), rows * k, k, _TYPE[dx_dtype], 0) if want_dx else _NO_MAT
    mw = (dw.data_ptr(), n * k, k, _TYPE[dw_dtype], 0) if want_dw else _NO_MAT
    _run_with_space("lipz_linear_backward", "lipz_linear_backward_workspace", _S_LINEAR_BACKWARD,
                    (_S_LINEAR_BACKWARD.size, code, slope, 0, groups, rows, k, n, *mats, *mx, *mw,
                     db.data_ptr() if want_db else 0, n), dev, device)
    return dx, dw, db
