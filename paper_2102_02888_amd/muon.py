"""Orthogonalised (Muon) updates of a list of matrices (include/onebit.h).

``Matrices`` describes where the matrices lie in flat buffers, in the layout
of a ``Plan`` over the same sizes unless offsets say otherwise; a
``Muon`` object owns the buffers of a run, as ``State`` does for 1-bit Adam.
"""
import ctypes

import numpy as np
import torch

from ._native import call
from .embedding import _one_device
from .onebit import _GRAD_DTYPES, _stream

__all__ = ["Matrices", "Muon", "MUON_SCALE_NONE", "MUON_SCALE_SPECTRAL", "MUON_SCALE_RMS",
           "PRODUCTS_F32", "PRODUCTS_F16", "onebit_muon_step", "onebit_orthogonalize",
           "matrices_kernels", "products_for"]

# The ONEBIT_PRODUCTS_* and ONEBIT_MUON_SCALE_* constants.
PRODUCTS_F32 = 0
PRODUCTS_F16 = 1
MUON_SCALE_NONE = 0
MUON_SCALE_SPECTRAL = 1
MUON_SCALE_RMS = 2


def products_for(out_dtype):
    """The products of a call that names none: PRODUCTS_F32, whatever type the
    output has, so that a result is off by the rounding to its type alone.
    PRODUCTS_F16 takes about half as long over long lists and adds up to 1e-3
    (bfloat16 results of gradients at the BERT-Large shape: 1.69e-3 from the
    exact ones as a whole, where the type's rounding is 1.66e-3); it is the
    caller's to ask for."""
    return PRODUCTS_F32


def _int64_array(values, count, name):
    if values is None:
        return None, None
    a = np.ascontiguousarray(np.asarray(values, dtype=np.int64))
    if a.shape != (count,):
        raise ValueError("%s must have one entry per matrix" % name)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def matrices_kernels(shapes, products=PRODUCTS_F32):
    """Which kernels the calls over matrices of these shapes take: the tiles'
    side and the groups of waves that share a tile, of a step's three products
    ("gram": D, "poly": B, "next": X + B X), and the most "parts" of a tile of D.
    Needs no GPU."""
    rows, rp = _int64_array([r for r, _ in shapes], len(shapes), "shapes")
    cols, cp = _int64_array([c for _, c in shapes], len(shapes), "shapes")
    side, groups = (ctypes.c_int32 * 3)(), (ctypes.c_int32 * 3)()
    parts = ctypes.c_int32()
    call("onebit_matrices_kernels", rp, cp, len(shapes), int(products), side, groups,
         ctypes.byref(parts))
    out = {name: (side[k], groups[k]) for k, name in enumerate(("gram", "poly", "next"))}
    out["parts"] = parts.value
    return out


class Matrices:
    """Matrices inside flat buffers, with their device tables.

    shapes: (rows, columns) of each.  offsets: element where each begins
    (default: one after another, each at the next multiple of 64); lds:
    elements from row to row (default: the columns)."""

    def __init__(self, shapes, offsets=None, lds=None):
        shapes = [(int(r), int(c)) for r, c in shapes]
        n = len(shapes)
        rows, rp = _int64_array([s[0] for s in shapes], n, "shapes")
        cols, cp = _int64_array([s[1] for s in shapes], n, "shapes")
        off, op = _int64_array(offsets, n, "offsets")
        ld, lp = _int64_array(lds, n, "lds")
        h = ctypes.c_void_p()
        call("onebit_matrices_create", rp, cp, op, lp, n, ctypes.byref(h))
        self._h = h
        self.shapes = shapes
        self.lds = [int(v) for v in (ld if ld is not None else cols)]
        extent = ctypes.c_int64()
        offset = np.zeros(n, np.int64)
        self._bytes = {}
        for products in (PRODUCTS_F32, PRODUCTS_F16):
            nbytes = ctypes.c_size_t()
            call("onebit_matrices_info", h, products, ctypes.byref(extent),
                 offset.ctypes.data_as(ctypes.c_void_p), ctypes.byref(nbytes))
            self._bytes[products] = nbytes.value
        self.extent = extent.value
        self.offsets = [int(v) for v in offset]

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("matrices are closed")
        return self._h

    def view(self, flat, k):
        """Matrix k of a flat buffer, as a 2-D view."""
        return flat.as_strided(self.shapes[k], (self.lds[k], 1),
                               flat.storage_offset() + self.offsets[k])

    def workspace_bytes(self, products=PRODUCTS_F32):
        return self._bytes[products]

    def workspace(self, device, products=PRODUCTS_F32):
        """A workspace for calls with these products, and with the other kind:
        one serves calls that differ in them."""
        most = max(self._bytes[products], *self._bytes.values(), 256)
        return torch.empty(most, dtype=torch.uint8, device=device)

    def close(self):
        if self._h is not None:
            call("onebit_matrices_destroy", self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _flat(t, mats, name, dtype=None):
    """(pointer, type code) of a flat buffer that holds the matrices."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if (dtype is not None and t.dtype != dtype) or t.dtype not in _GRAD_DTYPES:
        raise TypeError("%s must be %s, got %s" % (name, dtype or "float32, bfloat16 or float16",
                                                   t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.numel() < mats.extent:
        raise ValueError("%s has %d elements; the matrices reach %d" % (name, t.numel(),
                                                                      mats.extent))
    return t.data_ptr(), _GRAD_DTYPES[t.dtype]


def _workspace(t, mats, products):
    if products not in mats._bytes:
        raise ValueError("products must be PRODUCTS_F32 or PRODUCTS_F16")
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise TypeError("workspace must be a contiguous GPU tensor")
    have = t.numel() * t.element_size()
    if have < mats._bytes[products]:
        raise ValueError("workspace has %d bytes; the call needs %d"
                         % (have, mats._bytes[products]))
    return t.data_ptr()


def _coefficients(values):
    if values is None:
        return None
    a, b, c = (float(v) for v in values)
    return (ctypes.c_float * 3)(a, b, c)


def onebit_orthogonalize(mats, grad, out, workspace, products=None, steps=5, eps=1e-7,
                         coefficients=None, stream=None):
    """out = the matrices of grad, orthogonalised by `steps` Newton-Schulz
    steps; out may be grad itself.  products: PRODUCTS_F32 (the default,
    whatever out's type) or PRODUCTS_F16."""
    if products is None:
        products = products_for(out.dtype if isinstance(out, torch.Tensor) else None)
    gp, gcode = _flat(grad, mats, "grad")
    op, ocode = _flat(out, mats, "out")
    wp = _workspace(workspace, mats, products)
    _one_device(grad, out, workspace)
    call("onebit_orthogonalize", mats.handle, gp, gcode, op, ocode, products, int(steps),
         _coefficients(coefficients), float(eps), wp, _stream(stream))


def onebit_muon_step(mats, x, m, grads, lr, momentum, workspace, nesterov=True, weight_decay=0.0,
                     scale=MUON_SCALE_SPECTRAL, products=PRODUCTS_F32, steps=5, eps=1e-7,
                     coefficients=None, stream=None):
    """One Muon step of the matrices of x: the mean of grads' rows, momentum m,
    orthogonalised update.  grads: one flat buffer, or [n, >= extent] rows.
    scale: MUON_SCALE_SPECTRAL, sqrt(max(1, rows / columns)), is for matrices
    with a row per output (y = W x); MUON_SCALE_RMS, 0.2 sqrt(max(rows,
    columns)), fits both ways of storing them."""
    xp, _ = _flat(x, mats, "x", torch.float32)
    mp, _ = _flat(m, mats, "m", torch.float32)
    if not isinstance(grads, torch.Tensor) or grads.dtype not in _GRAD_DTYPES:
        raise TypeError("grads must be a float32, bfloat16 or float16 tensor")
    if not grads.is_cuda:
        raise ValueError("grads must be a GPU tensor")
    if grads.dim() == 1:
        n, cols, ld = 1, grads.numel(), grads.numel()
    elif grads.dim() == 2:
        (n, cols), ld = grads.shape, grads.stride(0)
    else:
        raise ValueError("grads must be 1-D or 2-D")
    if n < 1 or cols < mats.extent:
        raise ValueError("grads is %s; the call needs rows of at least %d elements"
                         % (tuple(grads.shape), mats.extent))
    if (cols > 1 and grads.stride(-1) != 1) or (n > 1 and ld < mats.extent):
        raise ValueError("grads must have unit stride in its last dimension, and rows apart")
    wp = _workspace(workspace, mats, products)
    _one_device(x, m, grads, workspace)
    call("onebit_muon_step", mats.handle, xp, mp, grads.data_ptr(), _GRAD_DTYPES[grads.dtype], ld,
         n, float(lr), float(momentum), int(bool(nesterov)), float(weight_decay), int(scale),
         int(products), int(steps), _coefficients(coefficients), float(eps), wp, _stream(stream))


class Muon:
    """Buffers and settings of a Muon run over `mats` with n simulated
    workers: fill `x` (flat parameters) once and `grads` ([n, extent]) before
    each step()."""

    def __init__(self, mats, device, lr, momentum=0.95, nesterov=True, weight_decay=0.0,
                 scale=MUON_SCALE_SPECTRAL, n_workers=1, grad_dtype=torch.float32,
                 products=PRODUCTS_F32, steps=5, eps=1e-7, coefficients=None):
        self.mats = mats
        self.lr, self.momentum, self.nesterov = lr, momentum, nesterov
        self.weight_decay, self.scale = weight_decay, scale
        self.products, self.steps, self.eps, self.coefficients = products, steps, eps, coefficients
        D = (mats.extent + 63) // 64 * 64
        self.x = torch.zeros(D, dtype=torch.float32, device=device)
        self.m = torch.zeros(D, dtype=torch.float32, device=device)
        self.grads = torch.zeros((n_workers, D), dtype=grad_dtype, device=device)
        self.workspace = mats.workspace(device, products)

    def step(self, lr=None, stream=None):
        onebit_muon_step(self.mats, self.x, self.m, self.grads, self.lr if lr is None else lr,
                         self.momentum, self.workspace, nesterov=self.nesterov,
                         weight_decay=self.weight_decay, scale=self.scale, products=self.products,
                         steps=self.steps, eps=self.eps, coefficients=self.coefficients,
                         stream=stream)

    STATE_KEYS = ("x", "m")

    def state_dict(self):
        """Host copies of what a later step reads (CPU tensors)."""
        return {k: getattr(self, k).detach().cpu().clone() for k in self.STATE_KEYS}

    def load_state_dict(self, sd):
        for k in self.STATE_KEYS:
            dst, src = getattr(self, k), sd[k]
            if tuple(src.shape) != tuple(dst.shape) or src.dtype != dst.dtype:
                raise ValueError("%s: expected %s %s, got %s %s" % (
                    k, tuple(dst.shape), dst.dtype, tuple(src.shape), src.dtype))
            dst.copy_(src)
