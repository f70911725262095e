"""Thin ctypes binding over the AdamW entry points of libgswa.so (see include/adamw.h).

The functions carry the names of the C entry points.  Tensors are checked (type, size, device) before the call; a missing library
is an error, there is no fallback path.
"""
import ctypes

from . import gswa
from ._args import Call
from .gswa import GSWA_BF16, GSWA_F32, _check

EXPORTS = ("adamw_query_bytes", "adamw_plan", "adamw_norm", "adamw_step", "adamw_unpack")
ADAMW_SKIP_NONFINITE = 1
BLOCK = 256   # elements that share an exponent in 8-bit states; tensors start at multiples of it in adamw_unpack's outputs


class adamw_desc(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_float), ("state_bits", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("seed", ctypes.c_uint64)]


class adamw_tensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("p_dtype", ctypes.c_int32), ("g_dtype", ctypes.c_int32), ("weight_decay", ctypes.c_float)]
    _fields_ += [(k, ctypes.c_void_p) for k in ("p", "master", "g", "m", "v", "m_exp", "v_exp")]


class adamw_plan_t(ctypes.Structure):
    _fields_ = [("desc", adamw_desc), ("n_tensors", ctypes.c_int32), ("chunks", ctypes.c_int64), ("blocks", ctypes.c_int64),
                ("buffer", ctypes.c_void_p), ("check", ctypes.c_uint64)]


_ready = False


def lib():
    global _ready
    L = gswa.lib()
    if not _ready:
        vp, dp, tp, pp = ctypes.c_void_p, ctypes.POINTER(adamw_desc), ctypes.POINTER(adamw_tensor), ctypes.POINTER(adamw_plan_t)
        L.adamw_query_bytes.argtypes = [dp, tp, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        L.adamw_plan.argtypes = [dp, tp, ctypes.c_int32, vp, pp, vp]
        L.adamw_norm.argtypes = [pp, vp, vp]
        L.adamw_step.argtypes = [pp, vp, ctypes.c_float, vp, vp, ctypes.c_float, vp]
        L.adamw_unpack.argtypes = [pp, vp, vp, vp]
        for n in EXPORTS:
            getattr(L, n).restype = ctypes.c_int
        _ready = True
    return L


def make_desc(beta1=0.9, beta2=0.999, eps=1e-8, state_bits=32, flags=0, seed=0):
    return adamw_desc(beta1, beta2, eps, state_bits, flags, seed)


def _dtype(name, t):
    import torch
    code = {torch.float32: GSWA_F32, torch.bfloat16: GSWA_BF16}.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return code


def _list(desc, tensors, c):
    import torch
    state = torch.uint8 if desc.state_bits == 8 else torch.float32
    out = (adamw_tensor * len(tensors))()
    for i, part in enumerate(tensors):
        unknown = set(part) - {"p", "master", "g", "m", "v", "m_exp", "v_exp", "weight_decay"}
        if unknown:
            raise ValueError(f"tensor {i}: unknown fields {sorted(unknown)}")
        p, g, n = part["p"], part["g"], part["p"].numel()
        if g.numel() != n:
            raise ValueError(f"tensor {i}: {n} parameters, {g.numel()} gradients")
        need = {"p": (p.dtype, n), "g": (g.dtype, n), "m": (state, n), "v": (state, n)}
        if part.get("master") is not None:
            need["master"] = (torch.float32, n)
        if desc.state_bits == 8:
            need.update({k: (torch.uint8, -(-n // BLOCK)) for k in ("m_exp", "v_exp")})
        places = {k: c.flat(f"{k} of tensor {i}", part[k], *need[k]) for k in need}
        out[i] = adamw_tensor(n, _dtype("p", p), _dtype("g", g), part.get("weight_decay", 0.0), **places)
    return out


class Plan:
    """A plan with what keeps its memory alive."""

    def __init__(self, tensors, buffer):
        self.c_plan, self.tensors, self.buffer = adamw_plan_t(), tensors, buffer

    @property
    def elements(self):
        """Elements of adamw_unpack's outputs."""
        return self.c_plan.blocks * BLOCK


def adamw_query_bytes(desc, tensors):
    """Bytes of a plan's buffer.  tensors: list of dicts with p, g, m, v and, where they apply, master, m_exp, v_exp, weight_decay."""
    n = ctypes.c_size_t()
    _check(lib().adamw_query_bytes(ctypes.byref(desc), _list(desc, tensors, Call()), len(tensors), ctypes.byref(n)))
    return n.value


def adamw_plan(desc, tensors, buffer, stream=None):
    """The Plan that the calls below take; it keeps the tensors and the buffer alive."""
    import torch
    L, c = lib(), Call()
    listed = _list(desc, tensors, c)
    n = ctypes.c_size_t()
    _check(L.adamw_query_bytes(ctypes.byref(desc), listed, len(tensors), ctypes.byref(n)))
    plan = Plan([dict(t) for t in tensors], buffer)
    c.run(L.adamw_plan, stream, ctypes.byref(desc), listed, len(tensors), c.flat("buffer", buffer, torch.uint8, n.value),
          ctypes.byref(plan.c_plan))
    return plan


def _call(plan):
    c = Call()
    c.device = plan.buffer.device
    return c


def adamw_norm(plan, norm, stream=None):
    import torch
    c = _call(plan)
    c.run(lib().adamw_norm, stream, ctypes.byref(plan.c_plan), c.flat("norm", norm, torch.float32, 1))


def adamw_step(plan, step, lr, lr_scale=None, norm=None, max_norm=0.0, stream=None):
    import torch
    c = _call(plan)
    c.run(lib().adamw_step, stream, ctypes.byref(plan.c_plan), c.flat("step", step, torch.int64, 1), lr,
          c.flat("lr_scale", lr_scale, torch.float32, 1), c.flat("norm", norm, torch.float32, 1), max_norm)


def adamw_unpack(plan, m_out, v_out, stream=None):
    import torch
    c = _call(plan)
    c.run(lib().adamw_unpack, stream, ctypes.byref(plan.c_plan), c.flat("m_out", m_out, torch.bfloat16, plan.elements),
          c.flat("v_out", v_out, torch.bfloat16, plan.elements))
