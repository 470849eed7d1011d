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


def _vector(t, name, width):
    """Pointer of a 1-D tensor of `width` elements side by side (None stays None)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype not in _GRAD_DTYPES:
        raise TypeError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.shape != (width,) or (width > 1 and t.stride(0) != 1):
        raise ValueError("%s must be 1-D with %d elements side by side, got %s with strides %s"
                         % (name, width, tuple(t.shape), t.stride()))
    return t.data_ptr()


def _pair(one, two, names, width):
    """(pointers, type code) of two such tensors that share a type."""
    pointers = _vector(one, names[0], width), _vector(two, names[1], width)
    if one is not None and two is not None and one.dtype != two.dtype:
        raise TypeError("%s and %s must be of one type, got %s and %s"
                        % (*names, one.dtype, two.dtype))
    given = two if one is None else one
    return pointers, 0 if given is None else _GRAD_DTYPES[given.dtype]


def onebit_layer_norm_forward(x, y, weight=None, bias=None, eps=1e-5, stream=None):
    """y = (x - mean) / sqrt(var + eps) * weight + bias of each row."""
    xp, xcode, xld, rows, width = _matrix(x, "x")
    yp, ycode, yld, _, _ = _matrix(y, "y", rows, width)
    (wp, bp), wcode = _pair(weight, bias, ("weight", "bias"), width)
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
    wp, wcode = _vector(weight, "weight", width), 0 if weight is None else _GRAD_DTYPES[weight.dtype]
    (dwp, dbp), dwcode = _pair(grad_weight, grad_bias, ("grad_weight", "grad_bias"), width)
    _one_device(*(t for t in (x, grad_y, grad_x, weight, grad_weight, grad_bias)
                  if t is not None))
    work = None
    if dwp is not None or dbp is not None:
        work = _workspace(workspace, "onebit_layer_norm_grad_workspace", rows, width)
    call("onebit_layer_norm_grad", yp, ycode, yld, xp, xcode, xld, rows, width, wp, wcode,
         float(eps), gp, gld, dwp, dbp, dwcode, int(bool(accumulate)), work, _stream(stream))
