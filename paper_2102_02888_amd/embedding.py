"""Token embedding on the flat buffers: lookup with scaling, and the table's
gradient by sorted tokens (include/onebit.h).

A table is any 2-D tensor with unit stride in its rows, such as a view into
the flat parameters, ``state.x[off:off + vocab * width].view(vocab, width)``;
its gradient likewise into a row of ``state.grads``.  Element types are
float32, bfloat16 and float16, in any combination; ids are int32 or int64.
"""
import ctypes

import torch

from ._native import call
from .onebit import _GRAD_DTYPES, _stream

__all__ = ["embedding_workspace", "onebit_embedding_forward", "onebit_embedding_grad"]

_ID_BYTES = {torch.int32: 4, torch.int64: 8}


def _matrix(t, name, rows=None, cols=None):
    """(pointer, type code, leading dimension, rows, columns) of a 2-D GPU
    tensor with unit stride in its rows; a contiguous tensor of more dimensions counts as rows
    of its last one."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    code = _GRAD_DTYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    shape = t.shape
    if len(shape) == 2:
        have, width = shape
        ld, unit = t.stride()
        if width > 1 and unit != 1:
            raise ValueError("%s must have unit stride in its last dimension" % name)
        if have > 1 and ld < width:
            raise ValueError("%s has overlapping rows" % name)
    elif len(shape) > 2 and t.is_contiguous():
        width = ld = shape[-1]
        have = t.numel() // width if width else 0
    else:
        raise ValueError("%s must be 2-D, or contiguous with more dimensions" % name)
    if (rows is not None and have != rows and shape[-1]) or (cols is not None and width != cols):
        raise ValueError("%s is %s; the call needs %s row(s) of %s elements"
                         % (name, tuple(shape), "any number of" if rows is None else rows, cols))
    return t.data_ptr(), code, ld if ld > width else width, have, width


def _ids(ids):
    """(pointer, bytes of an id, number of places)."""
    if not isinstance(ids, torch.Tensor) or ids.dtype not in _ID_BYTES:
        raise TypeError("ids must be an int32 or int64 tensor")
    if not ids.is_cuda:
        raise ValueError("ids must be a GPU tensor")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return ids.data_ptr(), _ID_BYTES[ids.dtype], ids.numel()


def _workspace(workspace, size, *sizes):
    """Pointer of a workspace that holds what the call named `size` says."""
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda \
            or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous GPU tensor")
    _one_device(workspace)
    need = ctypes.c_size_t()
    call(size, *sizes, ctypes.byref(need))
    if workspace.numel() * workspace.element_size() < need.value:
        raise ValueError("workspace has %d bytes; the call needs %d"
                         % (workspace.numel() * workspace.element_size(), need.value))
    return workspace.data_ptr()


def _one_device(*tensors):
    """The calls run on the current device, where all tensors have to be."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t.get_device() != here:
            raise ValueError("a tensor is on %s, the current device is cuda:%d" % (t.device, here))


def onebit_embedding_forward(table, ids, out, scale=1.0, stream=None):
    """out[t] = scale * table[ids[t]]; an id outside the table gives a row of
    zeros.  out: one row per id."""
    ip, ib, tokens = _ids(ids)
    tp, tcode, tld, vocab, width = _matrix(table, "table")
    op, ocode, old, _, _ = _matrix(out, "out", tokens, width)
    _one_device(table, ids, out)
    call("onebit_embedding_forward", tp, tcode, tld, vocab, width, ip, ib, tokens, float(scale),
         op, ocode, old, _stream(stream))


def embedding_workspace(tokens, vocab, width, device):
    """Workspace of onebit_embedding_grad for at most this many ids."""
    n = ctypes.c_size_t()
    call("onebit_embedding_grad_workspace", int(tokens), int(vocab), int(width), ctypes.byref(n))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def onebit_embedding_grad(grad_out, ids, grad_table, workspace, scale=1.0, padding_idx=-1,
                          accumulate=False, stream=None):
    """grad_table[v] = scale * sum of grad_out[t] over ids[t] == v, for every
    row v (accumulate: added to it); ids outside the table and equal to
    padding_idx add nothing."""
    ip, ib, tokens = _ids(ids)
    gp, gcode, gld, vocab, width = _matrix(grad_table, "grad_table")
    if grad_table.dim() != 2:
        raise ValueError("grad_table must be 2-D")
    dp, dcode, dld, _, _ = _matrix(grad_out, "grad_out", tokens, width)
    _one_device(grad_out, ids, grad_table)
    work = _workspace(workspace, "onebit_embedding_grad_workspace", tokens, vocab, width)
    call("onebit_embedding_grad", dp, dcode, dld, ip, ib, tokens, vocab, width,
         int(-1 if padding_idx is None else padding_idx), float(scale), gp, gcode, gld,
         int(bool(accumulate)), work, _stream(stream))
