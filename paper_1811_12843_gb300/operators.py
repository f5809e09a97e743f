"""The operators of a pre-norm residual block on torch tensors (C ABI: include/lipz.h).

    h, s = rmsnorm(x + s)          a = act(h W1^T + b1)          s' = a W2^T + b2 + s

forward and backward in bf16, and forward over 8-bit operands, for one network or for a population
of them: tensors are [rows, columns], or [groups, rows, columns] with weights per group. Columns
must be adjacent; rows and groups may be strided, and a group stride of 0 (``expand``) shares an
input between the groups. An output may not overlap an input unless its call says so (refused where
the strides show it). Every call runs the library's CUDA kernels on the current stream of the
tensors' device, allocates its outputs as torch does, waits for nothing, and may be captured in a
CUDA graph. What the library does not take raises ``LipzError`` with nothing launched. Nothing here
records an autograd graph: the backward passes are calls of their own, and a tensor that requires a
gradient is taken under ``torch.no_grad()`` or detached (else refused, since its gradient would be lost).
"""

import importlib.util
import os
import struct
from typing import NamedTuple, Optional

import torch

from . import LIPZ_ERR_INVALID, LipzError, library_path, load

__all__ = ["Norm", "rmsnorm", "rmsnorm_backward", "quantize_rows", "linear", "linear_backward",
           "ACTIVATIONS"]

ACTIVATIONS = {"none": 0, "relu": 1, "lrelu": 2, "tanh": 3, "gelu": 4, "silu": 5}

# the argument structures of include/lipz.h, which the binding must have been compiled with
_MAT, _VEC = "QqqiI", "Qq"
_S_RMSNORM = struct.Struct("=If3q" + 4 * _MAT + 3 * _VEC)
_S_RMSNORM_BACKWARD = struct.Struct("=II3q" + 4 * _MAT + 3 * _VEC + "QQ")
_S_QUANTIZE = struct.Struct("=II3q" + 2 * _MAT + _VEC)
_S_LINEAR = struct.Struct("=IifI4q" + 5 * _MAT + 3 * _VEC + "QQ")
_S_LINEAR_BACKWARD = struct.Struct("=IifI4q" + 6 * _MAT + _VEC + "QQ")
_STRUCTURES = (_S_RMSNORM, _S_RMSNORM_BACKWARD, _S_QUANTIZE, _S_LINEAR, _S_LINEAR_BACKWARD)

_module = None


def _load():
    """The compiled binding (csrc/torch_operators.cpp), which checks a call's tensors, allocates its
    results and makes the library's call."""
    global _module
    if _module is None:
        load()
        path = os.path.join(os.path.dirname(library_path()), "torch_operators.so")
        if not os.path.exists(path):
            raise LipzError(LIPZ_ERR_INVALID, "torch_operators.so is not built (%s); run "
                            "python -m paper_1811_12843_gb300._build" % path)
        spec = importlib.util.spec_from_file_location("torch_operators", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        if module.SIZES != tuple(s.size for s in _STRUCTURES):
            raise LipzError(LIPZ_ERR_INVALID, "%s was built for other argument structures" % path)
        _module = module
    return _module


def _act(call, act):
    code = ACTIVATIONS.get(act)
    if code is None:
        raise LipzError(LIPZ_ERR_INVALID, "%s: act must be one of %s (got %r)"
                        % (call, ", ".join(ACTIVATIONS), act))
    return code


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
    return Norm._make((_module or _load()).rmsnorm(x, weight, residual, eps, e4m3, keep, sum_out))


def rmsnorm_backward(dy, s, rstd, weight, dsum=None, want_dweight=True):
    """(dx, dweight) of rmsnorm: from its ``sum`` and ``rstd``, y's gradient, and dsum, the gradient
    that reaches the sum from elsewhere. dx is the gradient of x and of residual; dweight is fp32."""
    return (_module or _load()).rmsnorm_backward(dy, s, rstd, weight, dsum, want_dweight)


def quantize_rows(x):
    """(q, scale): x [.., rows, columns] (bf16 or fp32) in float8_e4m3fn with an fp32 scale per row,
    q scale the values."""
    return (_module or _load()).quantize_rows(x)


def linear(x, w, bias=None, act="none", slope=0.2, residual=None, x_scale=None, w_scale=None,
           out_dtype=torch.bfloat16, keep=False, out=None):
    """(y, pre): u = x w^T (x_scale[row] w_scale[column]) + bias, y = act(u) + residual.

    x [.., rows, k] and w [.., n, k]: bf16, or float8_e4m3fn with both scales; bias fp32; residual and
    y: out_dtype (bf16 or fp32). y is written to ``out`` if given (it may be the residual). ``keep``:
    pre is u in bf16, which the backward pass reads (else None)."""
    return (_module or _load()).linear(x, w, bias, _act("linear", act), slope, residual, x_scale, w_scale,
                                       out_dtype, keep, out)


def linear_backward(dy, x, w, act="none", slope=0.2, pre=None, want_dx=True, want_dw=True,
                    want_db=True, dx_dtype=torch.bfloat16, dw_dtype=torch.bfloat16):
    """(dx, dw, db) of linear over bf16 operands: du = dy act'(pre), dx = du w, dw = du^T x, db the
    sums of du over the rows (fp32); None for what is not wanted. dx and dw: bf16 or fp32. The
    residual's gradient is dy."""
    return (_module or _load()).linear_backward(dy, x, w, _act("linear_backward", act), slope, pre,
                                                want_dx, want_dw, want_db, dx_dtype, dw_dtype)
