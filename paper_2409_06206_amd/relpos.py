"""Thin ctypes binding over the relative-position-bias entry points of libgswa.so (see include/relpos.h).

The functions carry the names of the C entry points.  Tensors are checked against the descriptor (type, size, stride, device)
before the call; a missing library is an error, there is no fallback path.
"""
import ctypes

import torch

from . import gswa
from ._args import DTYPES, Call, Specs, Whole, row_spec, torch_dtype
from .gswa import GSWA_OK, _check

EXPORTS = ("relpos_log_edges", "relpos_query_bytes", "relpos_forward", "relpos_backward")
RELPOS_BIDIRECTIONAL, RELPOS_CAUSAL, RELPOS_ACCUM_WGRAD = 1, 2, 4
RELPOS_MAX_EDGES = 127


class relpos_desc(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32), ("window", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("q_len", ctypes.c_int32), ("k_len", ctypes.c_int32), ("q_start", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("n_edges", ctypes.c_int32), ("edges", ctypes.c_int32 * RELPOS_MAX_EDGES)]

    @property
    def buckets(self):
        """Rows of the learned table."""
        side = (self.n_edges + 1) * (2 if self.flags & RELPOS_BIDIRECTIONAL else 1)
        return side * side if self.window else side


_ready = False


def lib():
    global _ready
    L = gswa.lib()
    if not _ready:
        vp, ip, dp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(relpos_desc)
        L.relpos_log_edges.argtypes = [ctypes.c_int32] * 3 + [ip, ip]
        L.relpos_log_edges.restype = ctypes.c_int
        L.relpos_query_bytes.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        L.relpos_query_bytes.restype = ctypes.c_int
        L.relpos_forward.argtypes = [dp, vp, vp, vp]
        L.relpos_forward.restype = ctypes.c_int
        L.relpos_backward.argtypes = [dp] + [vp] * 4
        L.relpos_backward.restype = ctypes.c_int
        _ready = True
    return L


def relpos_log_edges(buckets, max_distance, bidirectional):
    """List of edges: single distances first, then even steps of the logarithm up to max_distance."""
    n, edges = ctypes.c_int32(), (ctypes.c_int32 * RELPOS_MAX_EDGES)()
    for v in (buckets, max_distance):
        if ctypes.c_int32(v).value != v:
            raise ValueError(f"32 bits cannot hold {v}")
    _check(lib().relpos_log_edges(buckets, max_distance, int(bool(bidirectional)), ctypes.byref(n), edges))
    return list(edges[: n.value])


_whole = Whole(relpos_desc)


def make_desc(heads, edges, dtype, flags=0, q_len=0, k_len=0, q_start=0, batch=1, window=0, row_stride=0):
    """Sequence form with q_len and k_len, window form with window."""
    if len(edges) > RELPOS_MAX_EDGES:
        raise ValueError(f"{len(edges)} edges, at most {RELPOS_MAX_EDGES}")
    code, n, places = DTYPES.get(dtype, dtype), len(edges), (ctypes.c_int32 * RELPOS_MAX_EDGES)(*edges)
    if places[:n] != list(edges):
        raise ValueError(f"edges cannot hold {[e for e, p in zip(edges, places) if e != p]}")
    return _whole.held(relpos_desc(heads, code, flags, window, batch, q_len, k_len, q_start, row_stride, n, places),
                       heads, code, flags, window, batch, q_len, k_len, q_start, row_stride, n)


def relpos_query_bytes(desc):
    """Scratch of relpos_backward in bytes."""
    n = ctypes.c_size_t()
    _check(lib().relpos_query_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def _spec(desc):
    """Types, elements of the table, what the bias and its gradient have to be (a number of elements, or rows), scratch."""
    n, t, ld = ctypes.c_size_t(), torch_dtype(desc.dtype), desc.row_stride or desc.k_len
    known = lib().relpos_query_bytes(ctypes.byref(desc), ctypes.byref(n)) == GSWA_OK   # (a descriptor that is none is refused by the call)
    if desc.window:
        bias = grad = (2 * desc.window - 1) ** 2 * desc.heads
    else:
        rows = desc.heads * desc.q_len
        bias, grad = (k * rows * desc.k_len if ld == desc.k_len else row_spec(k * rows, desc.k_len, ld) for k in (1, desc.batch))
    return t, torch.float32 if desc.window else t, desc.buckets * desc.heads, bias, grad, n.value if known else 0


_specs = Specs(_spec)


def _bias(c, name, t, dtype, spec):
    return c.flat(name, t, dtype, spec) if spec.__class__ is int else c.rows(name, t, dtype, spec)


def relpos_forward(desc, table, out, stream=None):
    t, _, n, bias, _, _ = _specs.of(desc)
    c = Call()
    c.run(gswa.lib().relpos_forward, stream, ctypes.byref(desc), c.flat("table", table, t, n), _bias(c, "out", out, t, bias))


def relpos_backward(desc, dout, dtable, ws, stream=None):
    """ws may be None where relpos_query_bytes is 0."""
    _, t, n, _, grad, need = _specs.of(desc)
    c = Call()
    c.run(gswa.lib().relpos_backward, stream, ctypes.byref(desc), _bias(c, "dout", dout, t, grad), c.flat("dtable", dtable, torch.float32, n),
          c.flat("ws", ws, torch.uint8, need))
