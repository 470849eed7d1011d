"""Layer norm of rows and its gradients (include/onebit.h).

Weight and bias are 1-D tensors of one element type, such as views into the
flat parameters, ``state.x[off:off + width]``; their gradients likewise into a
row of ``state.grads``.  Element types are float32, bfloat16 and float16.
"""
import ctypes

import torch

from ._native import call
from .embedding import _matrix, _one_device, _workspace
from .onebit import _GRAD_DTYPES, _stream

__all__ = ["layer_norm_workspace", "onebit_layer_norm_forward", "onebit_layer_norm_grad"]


def _vectors(width, **named):
    """(pointers, type code) of 1-D tensors of `width` elements that share a
    type; None stays None."""
    pointers, dtype = [], None
    for name, t in named.items():
        if t is None:
            pointers.append(None)
            continue
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dtype not in _GRAD_DTYPES or dtype not in (None, t.dtype):
            raise TypeError("%s must be float32, bfloat16 or float16, and of one type, got %s"
                            % (" and ".join(named), t.dtype))
        if not t.is_cuda:
            raise ValueError("%s must be a GPU tensor" % name)
        if t.dim() != 1 or t.shape[0] != width or (width > 1 and t.stride(0) != 1):
            raise ValueError("%s must be 1-D with %d elements side by side, got %s with strides %s"
                             % (name, width, tuple(t.shape), t.stride()))
        dtype = t.dtype
        pointers.append(t.data_ptr())
    return pointers, _GRAD_DTYPES.get(dtype, 0)


def onebit_layer_norm_forward(x, y, weight=None, bias=None, eps=1e-5, stream=None):
    """y = (x - mean) / sqrt(var + eps) * weight + bias of each row."""
    xp, xcode, xld, rows, width = _matrix(x, "x")
    yp, ycode, yld, _, _ = _matrix(y, "y", rows, width)
    (wp, bp), wcode = _vectors(width, weight=weight, bias=bias)
    _one_device(*(t for t in (x, y, weight, bias) if t is not None))
    call("onebit_layer_norm_forward", xp, xcode, xld, rows, width, wp, bp, wcode, float(eps), yp,
         ycode, yld, _stream(stream))


def layer_norm_workspace(rows, width, device):
    """Workspace of onebit_layer_norm_grad for at most this many rows and columns."""
    n = ctypes.c_size_t()
    call("onebit_layer_norm_grad_workspace", int(rows), int(width), ctypes.byref(n))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def onebit_layer_norm_grad(grad_y, x, grad_x, workspace, weight=None, grad_weight=None,
                           grad_bias=None, eps=1e-5, accumulate=False, stream=None):
    """The gradients of onebit_layer_norm_forward: grad_x (of x's type), and over
    all rows grad_weight and grad_bias (accumulate: added to them).  Any of the
    three may be None, and the workspace where the last two are."""
    xp, xcode, xld, rows, width = _matrix(x, "x")
    yp, ycode, yld, _, _ = _matrix(grad_y, "grad_y", rows, width)
    gp, gld = None, width
    if grad_x is not None:
        gp, gcode, gld, _, _ = _matrix(grad_x, "grad_x", rows, width)
        if gcode != xcode:
            raise TypeError("grad_x must be of x's type %s, got %s" % (x.dtype, grad_x.dtype))
    (wp,), wcode = _vectors(width, weight=weight)
    (dwp, dbp), dwcode = _vectors(width, grad_weight=grad_weight, grad_bias=grad_bias)
    _one_device(*(t for t in (x, grad_y, grad_x, weight, grad_weight, grad_bias)
                  if t is not None))
    work = None
    if dwp is not None or dbp is not None:
        work = _workspace(workspace, "onebit_layer_norm_grad_workspace", rows, width)
    call("onebit_layer_norm_grad", yp, ycode, yld, xp, xcode, xld, rows, width, wp, wcode,
         float(eps), gp, gld, dwp, dbp, dwcode, int(bool(accumulate)), work, _stream(stream))
