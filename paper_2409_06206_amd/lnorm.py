"""Thin ctypes binding over the LayerNorm entry points of libgswa.so (see include/lnorm.h).

The functions carry the names of the C entry points.  Tensors are checked against the descriptor (type, rows, stride, device)
before the call; a missing library is an error, there is no fallback path.
"""
import ctypes

import torch

from . import gswa
from ._args import DTYPES, Call, Specs, Whole, row_spec, torch_dtype
from .gswa import GSWA_OK, _check

EXPORTS = ("lnorm_query_bytes", "lnorm_forward", "lnorm_backward")
LNORM_ACCUM_WGRAD = 1


class lnorm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("flags", ctypes.c_uint32), ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64),
                ("r_stride", ctypes.c_int64)]


_ready = False


def lib():
    global _ready
    L = gswa.lib()
    if not _ready:
        vp, dp = ctypes.c_void_p, ctypes.POINTER(lnorm_desc)
        L.lnorm_query_bytes.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        L.lnorm_query_bytes.restype = ctypes.c_int
        L.lnorm_forward.argtypes = [dp] + [vp] * 7
        L.lnorm_forward.restype = ctypes.c_int
        L.lnorm_backward.argtypes = [dp] + [vp] * 9
        L.lnorm_backward.restype = ctypes.c_int
        _ready = True
    return L


_whole = Whole(lnorm_desc)


def make_desc(rows, C, dtype, eps=1e-5, flags=0, x_stride=0, y_stride=0, r_stride=0):
    code = DTYPES.get(dtype, dtype)
    return _whole.held(lnorm_desc(rows, C, code, eps, flags, x_stride, y_stride, r_stride), rows, C, code, flags, x_stride, y_stride, r_stride)


def lnorm_query_bytes(desc):
    """Scratch of lnorm_backward in bytes."""
    n = ctypes.c_size_t()
    _check(lib().lnorm_query_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def _spec(desc):
    n, C = ctypes.c_size_t(), desc.C
    known = lib().lnorm_query_bytes(ctypes.byref(desc), ctypes.byref(n)) == GSWA_OK   # (a descriptor that is none is refused by the call)
    return (torch_dtype(desc.dtype), C, row_spec(desc.rows, C, desc.x_stride or C), row_spec(desc.rows, C, desc.y_stride or C),
            row_spec(desc.rows, C, desc.r_stride or C), n.value if known else 0)


_specs = Specs(_spec)


def lnorm_forward(desc, x, residual, gamma, beta, y, sum, stream=None):
    """residual and sum, gamma, beta may be None (see the header)."""
    t, C, rx, ry, rr, _ = _specs.of(desc)
    c = Call()
    c.run(gswa.lib().lnorm_forward, stream, ctypes.byref(desc), c.rows("x", x, t, rx), c.rows("residual", residual, t, rr),
          c.flat("gamma", gamma, t, C), c.flat("beta", beta, t, C), c.rows("y", y, t, ry), c.rows("sum", sum, t, rr))


def lnorm_backward(desc, x, dy, gamma, dsum, dx, dgamma, dbeta, ws, stream=None):
    """gamma, dsum, and dgamma with dbeta (and then ws) may be None."""
    t, C, rx, ry, rr, need = _specs.of(desc)
    c, f32 = Call(), torch.float32
    c.run(gswa.lib().lnorm_backward, stream, ctypes.byref(desc), c.rows("x", x, t, rx), c.rows("dy", dy, t, ry), c.flat("gamma", gamma, t, C),
          c.rows("dsum", dsum, t, rr), c.rows("dx", dx, t, rr), c.flat("dgamma", dgamma, f32, C), c.flat("dbeta", dbeta, f32, C),
          c.flat("ws", ws, torch.uint8, need))
