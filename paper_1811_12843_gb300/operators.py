"""The operators of a pre-norm residual block on torch tensors (C ABI: include/lipz.h).

    h, s = rmsnorm(x + s)          a = act(h W1^T + b1)          s' = a W2^T + b2 + s

forward and backward in bf16, and forward over 8-bit operands, for one network or for a population
of them: tensors are [rows, columns], or [groups, rows, columns] with weights per group. Columns
must be adjacent; rows and groups may be strided, and a group stride of 0 (``expand``) shares an
input between the groups. Every call runs the library's CUDA kernels on the current stream of the
tensors' device, allocates its outputs as torch does, waits for nothing, and may be captured in a
CUDA graph. What the library does not take raises ``LipzError`` with nothing launched. Nothing here
records an autograd graph: the backward passes are calls of their own.
"""

import struct
from typing import NamedTuple, Optional

import torch

from . import (LIPZ_BF16, LIPZ_E4M3, LIPZ_ERR_INVALID, LIPZ_FP32, LipzError, lipz_linear,
               lipz_linear_backward, lipz_linear_backward_workspace, lipz_linear_workspace,
               lipz_quantize_rows, lipz_rmsnorm, lipz_rmsnorm_backward,
               lipz_rmsnorm_backward_workspace)

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


def _refuse(call, what):
    raise LipzError(LIPZ_ERR_INVALID, "%s: %s" % (call, what))


def _mat(call, name, t, shape, dtypes, device):
    """(address, group stride, row stride, type, 0) of a checked matrix."""
    if t is None:
        return _NO_MAT
    if not isinstance(t, torch.Tensor) or t.device != device or not t.is_cuda:
        _refuse(call, "%s must be a CUDA tensor on the same device as the others" % name)
    if t.dtype not in dtypes:
        _refuse(call, "%s has dtype %s, taken are %s" % (name, t.dtype, ", ".join(map(str, dtypes))))
    if t.shape != shape:
        _refuse(call, "%s has shape %s, not %s" % (name, list(t.shape), list(shape)))
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1 and t.numel():
        _refuse(call, "%s: columns must be adjacent" % name)
    return t.data_ptr(), st[0] if len(st) == 3 else 0, st[-2], _TYPE[t.dtype], 0


def _vec(call, name, t, shape, device):
    """(address, group stride) of a checked fp32 vector."""
    if t is None:
        return _NO_VEC
    if not isinstance(t, torch.Tensor) or t.device != device or not t.is_cuda:
        _refuse(call, "%s must be a CUDA tensor on the same device as the others" % name)
    if t.dtype is not _F32 or t.shape != shape:
        _refuse(call, "%s must be float32 of shape %s, not %s of %s"
                % (name, list(shape), t.dtype, list(t.shape)))
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1 and t.numel():
        _refuse(call, "%s: elements must be adjacent" % name)
    return t.data_ptr(), st[0] if len(st) == 2 else 0


def _first(call, name, t):
    """(leading dimensions, groups, rows, columns, device) that a call's other tensors go by."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() not in (2, 3):
        _refuse(call, "%s must be a CUDA tensor [rows, columns] or [groups, rows, columns]" % name)
    s = t.shape
    return s[:-2], (s[0] if len(s) == 3 else 1), s[-2], s[-1], t.device


def _act(call, act):
    code = ACTIVATIONS.get(act)
    if code is None:
        _refuse(call, "act must be one of %s (got %r)" % (", ".join(ACTIVATIONS), act))
    return code


def _run(f, args, device):
    """The call on the device's current stream."""
    stream = torch.cuda.current_stream(device).cuda_stream
    if device.index == torch.cuda.current_device():
        return f(args, stream)
    with torch.cuda.device(device):
        return f(args, stream)


def _run_with_space(f, space, pack, fields, device):
    """The call with the workspace that it asks for."""
    args = pack(*fields, 0, 0)
    if device.index == torch.cuda.current_device():
        need = space(args)
    else:
        with torch.cuda.device(device):
            need = space(args)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=device)
        args = pack(*fields, work.data_ptr(), need)
    return _run(f, args, device)


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
    lead, groups, rows, dim, dev = _first(call, "x", x)
    shape, dt = x.shape, (x.dtype,)
    mx = _mat(call, "x", x, shape, (_BF16, _F32), dev)
    mr = _mat(call, "residual", residual, shape, dt, dev)
    vw = _vec(call, "weight", weight, lead + (dim,), dev)
    if residual is None:
        if sum_out is not None:
            _refuse(call, "sum_out needs a residual")
        total, ms = x, _NO_MAT
    else:
        total = torch.empty(shape, dtype=x.dtype, device=dev) if sum_out is None else sum_out
        ms = _mat(call, "sum_out", total, shape, dt, dev)
    y = torch.empty(shape, dtype=_E4M3 if e4m3 else x.dtype, device=dev)
    scale = torch.empty(lead + (rows,), dtype=_F32, device=dev) if e4m3 else None
    rstd = torch.empty(lead + (rows,), dtype=_F32, device=dev) if keep else None
    args = _S_RMSNORM.pack(
        _S_RMSNORM.size, eps, groups, rows, dim, *mx, *mr, *ms,
        y.data_ptr(), rows * dim, dim, LIPZ_E4M3 if e4m3 else _TYPE[x.dtype], 0, *vw,
        scale.data_ptr() if e4m3 else 0, rows, rstd.data_ptr() if keep else 0, rows)
    _run(lipz_rmsnorm, args, dev)
    return Norm(y, total, scale, rstd)


def rmsnorm_backward(dy, s, rstd, weight, dsum=None, want_dweight=True):
    """(dx, dweight) of rmsnorm: from its ``sum`` and ``rstd``, y's gradient, and dsum, the gradient
    that reaches the sum from elsewhere. dx is the gradient of x and of residual; dweight is fp32."""
    call = "rmsnorm_backward"
    lead, groups, rows, dim, dev = _first(call, "s", s)
    shape, dt = s.shape, (s.dtype,)
    mats = (_mat(call, "dy", dy, shape, dt, dev) + _mat(call, "s", s, shape, (_BF16, _F32), dev)
            + _mat(call, "dsum", dsum, shape, dt, dev))
    if dy is None:
        _refuse(call, "dy must be given")
    vecs = (_vec(call, "weight", weight, lead + (dim,), dev)
            + _vec(call, "rstd", rstd, lead + (rows,), dev))
    dx = torch.empty(shape, dtype=s.dtype, device=dev)
    dweight = torch.empty(lead + (dim,), dtype=_F32, device=dev) if want_dweight else None
    fields = (_S_RMSNORM_BACKWARD.size, 0, groups, rows, dim, *mats, dx.data_ptr(), rows * dim, dim,
              _TYPE[s.dtype], 0, *vecs, dweight.data_ptr() if want_dweight else 0, dim)
    _run_with_space(lipz_rmsnorm_backward, lipz_rmsnorm_backward_workspace, _S_RMSNORM_BACKWARD.pack,
                    fields, dev)
    return dx, dweight


def quantize_rows(x):
    """(q, scale): x [.., rows, columns] (bf16 or fp32) in float8_e4m3fn with an fp32 scale per row,
    q scale the values."""
    call = "quantize_rows"
    lead, groups, rows, dim, dev = _first(call, "x", x)
    mx = _mat(call, "x", x, x.shape, (_BF16, _F32), dev)
    q = torch.empty(x.shape, dtype=_E4M3, device=dev)
    scale = torch.empty(lead + (rows,), dtype=_F32, device=dev)
    _run(lipz_quantize_rows,
         _S_QUANTIZE.pack(_S_QUANTIZE.size, 0, groups, rows, dim, *mx, q.data_ptr(), rows * dim, dim,
                          LIPZ_E4M3, 0, scale.data_ptr(), rows), dev)
    return q, scale


def linear(x, w, bias=None, act="none", slope=0.2, residual=None, x_scale=None, w_scale=None,
           out_dtype=torch.bfloat16, keep=False, out=None):
    """(y, pre): u = x w^T (x_scale[row] w_scale[column]) + bias, y = act(u) + residual.

    x [.., rows, k] and w [.., n, k]: bf16, or float8_e4m3fn with both scales; bias fp32; residual and
    y: out_dtype (bf16 or fp32). y is written to ``out`` if given (it may be the residual). ``keep``:
    pre is u in bf16, which the backward pass reads (else None)."""
    call = "linear"
    lead, groups, rows, k, dev = _first(call, "x", x)
    if not isinstance(w, torch.Tensor) or w.dim() != x.dim():
        _refuse(call, "w must be a CUDA tensor with x's number of dimensions")
    n = w.shape[-2]
    shape = lead + (rows, n)
    code = _act(call, act)
    if out_dtype not in (_BF16, _F32):
        _refuse(call, "out_dtype must be bfloat16 or float32")
    mx = _mat(call, "x", x, x.shape, (_BF16, _E4M3), dev)
    mw = _mat(call, "w", w, lead + (n, k), (x.dtype,), dev)
    mr = _mat(call, "residual", residual, shape, (out_dtype,), dev)
    if (x_scale is None) != (x.dtype is not _E4M3) or (w_scale is None) != (x.dtype is not _E4M3):
        _refuse(call, "x_scale and w_scale go with 8-bit operands, and with them alone")
    vecs = (_vec(call, "x_scale", x_scale, lead + (rows,), dev)
            + _vec(call, "w_scale", w_scale, lead + (n,), dev)
            + _vec(call, "bias", bias, lead + (n,), dev))
    y = torch.empty(shape, dtype=out_dtype, device=dev) if out is None else out
    my = _mat(call, "out", y, shape, (out_dtype,), dev)
    pre = torch.empty(shape, dtype=_BF16, device=dev) if keep else None
    mp = (pre.data_ptr(), rows * n, n, LIPZ_BF16, 0) if keep else _NO_MAT
    fields = (_S_LINEAR.size, code, slope, 0, groups, rows, k, n, *mx, *mw, *mr, *my, *mp, *vecs)
    _run_with_space(lipz_linear, lipz_linear_workspace, _S_LINEAR.pack, fields, dev)
    return y, pre


def linear_backward(dy, x, w, act="none", slope=0.2, pre=None, want_dx=True, want_dw=True,
                    want_db=True, dw_dtype=torch.bfloat16):
    """(dx, dw, db) of linear over bf16 operands: du = dy act'(pre), dx = du w, dw = du^T x, db the
    sums of du over the rows; None for what is not wanted. The residual's gradient is dy."""
    call = "linear_backward"
    lead, groups, rows, n, dev = _first(call, "dy", dy)
    if not isinstance(x, torch.Tensor) or x.dim() != dy.dim():
        _refuse(call, "x must be a CUDA tensor with dy's number of dimensions")
    k = x.shape[-1]
    code = _act(call, act)
    if code and pre is None:
        _refuse(call, "act %r needs pre" % act)
    if dw_dtype not in (_BF16, _F32):
        _refuse(call, "dw_dtype must be bfloat16 or float32")
    bf = (_BF16,)
    mats = (_mat(call, "dy", dy, dy.shape, bf, dev) + _mat(call, "x", x, lead + (rows, k), bf, dev)
            + _mat(call, "w", w, lead + (n, k), bf, dev)
            + _mat(call, "pre", pre if code else None, dy.shape, bf, dev))
    if w is None:
        _refuse(call, "w must be given")
    dx = torch.empty(lead + (rows, k), dtype=_BF16, device=dev) if want_dx else None
    dw = torch.empty(lead + (n, k), dtype=dw_dtype, device=dev) if want_dw else None
    db = torch.empty(lead + (n,), dtype=_F32, device=dev) if want_db else None
    fields = (_S_LINEAR_BACKWARD.size, code, slope, 0, groups, rows, k, n, *mats,
              *((dx.data_ptr(), rows * k, k, LIPZ_BF16, 0) if want_dx else _NO_MAT),
              *((dw.data_ptr(), n * k, k, _TYPE[dw_dtype], 0) if want_dw else _NO_MAT),
              db.data_ptr() if want_db else 0, n)
    _run_with_space(lipz_linear_backward, lipz_linear_backward_workspace, _S_LINEAR_BACKWARD.pack,
                    fields, dev)
    return dx, dw, db
