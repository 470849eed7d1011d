"""What a language model's logits are turned into (include/onebit.h): the
log-probabilities of given tokens with entropies and top alternatives, and the
divergence from a teacher's top logits, each with the logits' gradient.

Logits are any 2-D tensor with unit stride in its rows (or contiguous with more
dimensions: rows of the last one), of float32, bfloat16 or float16; a gradient
has the logits' type and may be written over them.  Values of a row are float32.
"""
import torch

from ._native import call
from .embedding import _ids, _matrix, _one_device
from .onebit import _stream

__all__ = ["onebit_distill_forward", "onebit_distill_grad", "onebit_logprobs_forward",
           "onebit_logprobs_grad"]


def _values(t, name, count):
    """Pointer of a contiguous float32 tensor of `count` elements (None stays None)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32:
        raise TypeError("%s must be a float32 tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if not t.is_contiguous() or t.numel() != count:
        raise ValueError("%s must be contiguous with %d elements, got %s" % (name, count,
                                                                             tuple(t.shape)))
    return t.data_ptr()


def _row_ids(ids, rows, name="ids"):
    pointer, size, count = _ids(ids)
    if count != rows:
        raise ValueError("%s has %d elements; the call needs %d" % (name, count, rows))
    return pointer, size


def _gradient(grad, logits, rows, vocab, code):
    gp, gcode, gld, _, _ = _matrix(grad, "grad_logits", rows, vocab)
    if gcode != code:
        raise TypeError("grad_logits must be of the logits' type %s, got %s"
                        % (logits.dtype, grad.dtype))
    return gp, gld


def _here(*tensors):
    _one_device(*(t for t in tensors if t is not None))


def onebit_logprobs_forward(logits, ids, logprobs, scale=1.0, entropy=None, top_ids=None,
                            top_logprobs=None, stream=None):
    """logprobs[r] = log softmax(scale * logits[r]) at ids[r] (0 where that is not
    a token), entropy[r] of the row's distribution, and the top alternatives of
    each row in order: top_ids [rows, k] of ids' type and top_logprobs [rows, k],
    k up to 64.  Any output may be None, and ids where logprobs and top_ids are."""
    lp, code, ld, rows, vocab = _matrix(logits, "logits")
    tops = [t for t in (top_ids, top_logprobs) if t is not None]
    k = 0
    for t in tops:
        if not isinstance(t, torch.Tensor) or t.dim() < 1 or t.shape[-1] != tops[0].shape[-1]:
            raise ValueError("top_ids and top_logprobs must be tensors of as many columns")
        k = t.shape[-1]
    ip, ib, tp = None, 4, None
    if ids is not None:
        ip, ib = _row_ids(ids, rows)
    elif logprobs is not None:
        raise TypeError("ids must be an int32 or int64 tensor")
    if top_ids is not None:
        tp, tb = _row_ids(top_ids, rows * k, "top_ids")
        if ids is not None and tb != ib:
            raise TypeError("top_ids must be of ids' type %s, got %s" % (ids.dtype, top_ids.dtype))
        ib = tb
    vp, ep = _values(logprobs, "logprobs", rows), _values(entropy, "entropy", rows)
    tlp = _values(top_logprobs, "top_logprobs", rows * k)
    _here(logits, ids, logprobs, entropy, top_ids, top_logprobs)
    call("onebit_logprobs_forward", lp, code, ld, rows, vocab, ip, ib, float(scale), vp, ep, k,
         tp, tlp, _stream(stream))


def onebit_logprobs_grad(logits, ids, grad_logprobs, grad_logits, scale=1.0, grad_entropy=None,
                         logprobs=None, entropy=None, stream=None):
    """grad_logits = the gradient of the sum of grad_logprobs * logprobs +
    grad_entropy * entropy, zeros in rows whose id is not a token; logprobs and
    entropy are given too where they are not None.  grad_logits may be logits."""
    lp, code, ld, rows, vocab = _matrix(logits, "logits")
    ip, ib = _row_ids(ids, rows)
    gp, gld = _gradient(grad_logits, logits, rows, vocab, code)
    given = (_values(grad_logprobs, "grad_logprobs", rows),
             _values(grad_entropy, "grad_entropy", rows))
    wanted = _values(logprobs, "logprobs", rows), _values(entropy, "entropy", rows)
    _here(logits, ids, grad_logprobs, grad_logits, grad_entropy, logprobs, entropy)
    call("onebit_logprobs_grad", lp, code, ld, rows, vocab, ip, ib, float(scale), *given, gp, gld,
         *wanted, _stream(stream))


def _teacher(teacher_ids, teacher_logits, rows):
    tp, tcode, tld, _, k = _matrix(teacher_logits, "teacher_logits", rows)
    ip, ib = _row_ids(teacher_ids, rows * k, "teacher_ids")
    return ip, ib, tp, tcode, tld, k


def onebit_distill_forward(logits, teacher_ids, teacher_logits, loss, scale=1.0, stream=None):
    """loss[r] = the divergence of softmax(scale * logits[r]) from the teacher's
    softmax(scale * teacher_logits[r]) over its alternatives teacher_ids[r]
    (both [rows, k], k up to 256); alternatives that are not tokens are left out."""
    lp, code, ld, rows, vocab = _matrix(logits, "logits")
    teacher = _teacher(teacher_ids, teacher_logits, rows)
    vp = _values(loss, "loss", rows)
    _here(logits, teacher_ids, teacher_logits, loss)
    call("onebit_distill_forward", lp, code, ld, rows, vocab, *teacher, float(scale), vp,
         _stream(stream))


def onebit_distill_grad(logits, teacher_ids, teacher_logits, grad_loss, grad_logits, scale=1.0,
                        loss=None, stream=None):
    """grad_logits = the gradient of the sum of grad_loss * loss; the loss is given
    too where it is not None.  grad_logits may be logits."""
    lp, code, ld, rows, vocab = _matrix(logits, "logits")
    teacher = _teacher(teacher_ids, teacher_logits, rows)
    gp, gld = _gradient(grad_logits, logits, rows, vocab, code)
    wp, vp = _values(grad_loss, "grad_loss", rows), _values(loss, "loss", rows)
    _here(logits, teacher_ids, teacher_logits, grad_loss, grad_logits, loss)
    call("onebit_distill_grad", lp, code, ld, rows, vocab, *teacher, float(scale), wp, gp, gld, vp,
         _stream(stream))
