"""Attention over packed sequences and its gradients (include/onebit.h).

Queries, keys, values and results are [tokens, heads, dim] tensors of bfloat16 or
float16 whose heads lie side by side, such as parts of one projection's output,
``qkv.view(tokens, heads + 2 * kv_heads, dim).split([heads, kv_heads, kv_heads], 1)``.
``starts`` holds the sequences' first tokens and the last one's end (int32).
"""
import ctypes

import torch

from ._native import call
from .embedding import _one_device, _workspace
from .loss import _values
from .onebit import _GRAD_DTYPES, _stream

__all__ = ["attention_workspace", "onebit_attention_forward", "onebit_attention_grad"]


def _heads(t, name, like=None, shape=None):
    """(pointer, elements from token to token) of a [tokens, heads, dim] GPU tensor
    of q's type, and of the shape that the call needs."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype not in (torch.bfloat16, torch.float16) or (like is not None and t.dtype != like):
        raise TypeError("%s must be %s, got %s" % (name, "bfloat16 or float16" if like is None
                                                   else like, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.dim() != 3 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError("%s is %s; the call needs %s"
                         % (name, tuple(t.shape), shape or "[tokens, heads, dim]"))
    tokens, heads, dim = t.shape
    ld, head, unit = t.stride()
    if (dim > 1 and unit != 1) or (heads > 1 and head != dim):
        raise ValueError("%s must have its heads side by side, got strides %s" % (name, t.stride()))
    if tokens > 1 and ld < heads * dim:
        raise ValueError("%s has overlapping tokens" % name)
    return t.data_ptr(), max(ld, heads * dim)


def _starts(starts):
    """(pointer, number of sequences)."""
    if not isinstance(starts, torch.Tensor) or starts.dtype != torch.int32:
        raise TypeError("starts must be an int32 tensor")
    if not starts.is_cuda:
        raise ValueError("starts must be a GPU tensor")
    if starts.dim() != 1 or starts.numel() < 1 or not starts.is_contiguous():
        raise ValueError("starts must be 1-D and contiguous, one more than sequences")
    return starts.data_ptr(), starts.numel() - 1


def _inputs(q, k, v):
    qp, qld = _heads(q, "q")
    tokens, heads, dim = q.shape
    if not isinstance(k, torch.Tensor) or k.dim() != 3 or not k.shape[1] or heads % k.shape[1]:
        raise ValueError("k must be [tokens, kv_heads, dim], kv_heads a divisor of q's heads")
    shape = (tokens, k.shape[1], dim)
    kp, kld = _heads(k, "k", q.dtype, shape)
    vp, vld = _heads(v, "v", q.dtype, shape)
    return (qp, qld, kp, kld, vp, vld), shape


def onebit_attention_forward(q, k, v, starts, out, lse=None, causal=True, scale=None,
                             stream=None):
    """out = softmax(scale q k') v of each head over each sequence (causal: over the
    tokens up to the query's own); lse [tokens, heads] float32, for the gradient.
    scale: dim ** -0.5 unless given."""
    sides, _ = _inputs(q, k, v)
    tokens, heads, dim = q.shape
    op, old = _heads(out, "out", q.dtype, (tokens, heads, dim))
    lp = _values(lse, "lse", tokens * heads)
    sp, sequences = _starts(starts)
    _one_device(*(t for t in (q, k, v, starts, out, lse) if t is not None))
    call("onebit_attention_forward", *sides, _GRAD_DTYPES[q.dtype], tokens, heads, k.shape[1], dim,
         sp, sequences, int(bool(causal)), dim ** -0.5 if scale is None else float(scale), op, old,
         lp, _stream(stream))


def attention_workspace(tokens, heads, device):
    """Workspace of onebit_attention_grad for at most this many tokens and heads."""
    n = ctypes.c_size_t()
    call("onebit_attention_grad_workspace", int(tokens), int(heads), ctypes.byref(n))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def onebit_attention_grad(grad_out, q, k, v, out, lse, starts, grad_q, grad_k, grad_v, workspace,
                          causal=True, scale=None, stream=None):
    """The gradients of onebit_attention_forward's queries, keys and values; out and
    lse are its results.  They may be parts of one tensor."""
    sides, kv_shape = _inputs(q, k, v)
    shape = tokens, heads, dim = tuple(q.shape)
    dp, dld = _heads(grad_out, "grad_out", q.dtype, shape)
    op, old = _heads(out, "out", q.dtype, shape)
    lp = _values(lse, "lse", tokens * heads)
    grads = (*_heads(grad_q, "grad_q", q.dtype, shape), *_heads(grad_k, "grad_k", q.dtype, kv_shape),
             *_heads(grad_v, "grad_v", q.dtype, kv_shape))
    sp, sequences = _starts(starts)
    _one_device(*(t for t in (q, k, v, out, lse, starts, grad_out, grad_q, grad_k, grad_v)
                  if t is not None))
    work = _workspace(workspace, "onebit_attention_grad_workspace", tokens, heads)
    call("onebit_attention_grad", dp, dld, *sides, op, old, lp, _GRAD_DTYPES[q.dtype], tokens,
         heads, k.shape[1], dim, sp, sequences, int(bool(causal)),
         dim ** -0.5 if scale is None else float(scale), *grads, work, _stream(stream))
