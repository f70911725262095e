"""Thin ctypes binding over the AdamW entry points of libgswa.so (see include/adamw.h).

The functions carry the names of the C entry points.  Tensors are checked (type, size, device) before the call; a missing library
is an error, there is no fallback path.
"""
import ctypes
import struct

import torch

from . import gswa
from ._args import Call, Whole
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


_ROW = struct.Struct("@qiif4x7Q")   # an adamw_tensor: filled in one go, a list of some hundred tensors is as long as a step
assert _ROW.size == ctypes.sizeof(adamw_tensor)


class adamw_plan_t(ctypes.Structure):
    _fields_ = [("desc", adamw_desc), ("n_tensors", ctypes.c_int32), ("each", ctypes.c_int32), ("chunks", ctypes.c_int64), ("blocks", ctypes.c_int64),
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


_whole = Whole(adamw_desc)


def make_desc(beta1=0.9, beta2=0.999, eps=1e-8, state_bits=32, flags=0, seed=0):
    seed = int(seed) & 0xFFFFFFFFFFFFFFFF
    return _whole.held(adamw_desc(beta1, beta2, eps, state_bits, flags, seed), state_bits, flags, seed)


_FIELDS = frozenset(("p", "master", "g", "m", "v", "m_exp", "v_exp", "weight_decay"))
_CODES = {torch.float32: GSWA_F32, torch.bfloat16: GSWA_BF16}


def _list(desc, tensors):
    """The C list of tensors and the index of the device they lie on."""
    eight, f32, u8 = desc.state_bits == 8, torch.float32, torch.uint8
    state, device = u8 if eight else f32, None
    out = (adamw_tensor * len(tensors))()

    def place(name, t, dtype, n):
        if t.get_device() != device or t.dtype is not dtype or not t.is_contiguous() or t.numel() < n:
            raise ValueError(f"tensor {i}: {name} must be a contiguous tensor of at least {n} elements of {dtype} on GPU {device}, not {t.numel()} "
                             f"of {t.dtype} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")
        return t.data_ptr()

    for i, part in enumerate(tensors):
        if not _FIELDS.issuperset(part):
            raise ValueError(f"tensor {i}: unknown fields {sorted(set(part) - _FIELDS)}")
        p, g, master = part["p"], part["g"], part.get("master")
        n, p_code, g_code = p.numel(), _CODES.get(p.dtype), _CODES.get(g.dtype)
        if g.numel() != n:
            raise ValueError(f"tensor {i}: {n} parameters, {g.numel()} gradients")
        if p_code is None or g_code is None:
            raise ValueError(f"tensor {i}: parameters and gradients must be float32 or bfloat16, not {p.dtype} and {g.dtype}")
        if device is None:
            device = p.get_device()
            if device < 0:
                raise ValueError(f"tensor {i}: p must lie on a GPU")
        m_exp = v_exp = 0
        if eight:
            blocks = -(-n // BLOCK)
            m_exp, v_exp = place("m_exp", part["m_exp"], u8, blocks), place("v_exp", part["v_exp"], u8, blocks)
        _ROW.pack_into(out, i * _ROW.size, n, p_code, g_code, part.get("weight_decay", 0.0), place("p", p, p.dtype, n),
                       0 if master is None else place("master", master, f32, n), place("g", g, g.dtype, n),
                       place("m", part["m"], state, n), place("v", part["v"], state, n), m_exp, v_exp)
    return out, device


class Plan:
    """A plan with what keeps its memory alive."""

    def __init__(self, tensors, buffer):
        self.c_plan, self.tensors, self.buffer, self.device = adamw_plan_t(), tensors, buffer, buffer.get_device()
        self.c_ref = ctypes.byref(self.c_plan)

    @property
    def elements(self):
        """Elements of adamw_unpack's outputs."""
        return self.c_plan.blocks * BLOCK


def adamw_query_bytes(desc, tensors):
    """Bytes of a plan's buffer.  tensors: list of dicts with p, g, m, v and, where they apply, master, m_exp, v_exp, weight_decay."""
    n, sizes = ctypes.c_size_t(), (adamw_tensor * len(tensors))()
    for row, part in zip(sizes, tensors):
        row.n = part["p"].numel()
    _check(lib().adamw_query_bytes(ctypes.byref(desc), sizes, len(tensors), ctypes.byref(n)))
    return n.value


def adamw_plan(desc, tensors, buffer, stream=None):
    """The Plan that the calls below take; it keeps the tensors and the buffer alive.

    Checking and listing the tensors here takes some 2 us each (468 of them 1.1 ms, where norm and step take 16 us): a plan is made once for tensors
    that stay where they are, gradients too.  A program whose gradients are allocated anew each step would pay for it each step."""
    L, n = lib(), ctypes.c_size_t()
    listed, device = _list(desc, tensors)
    c = Call(device)
    _check(L.adamw_query_bytes(ctypes.byref(desc), listed, len(tensors), ctypes.byref(n)))
    plan = Plan([dict(t) for t in tensors], buffer)
    c.run(L.adamw_plan, stream, ctypes.byref(desc), listed, len(tensors), c.flat("buffer", buffer, torch.uint8, n.value),
          ctypes.byref(plan.c_plan))
    return plan


def adamw_norm(plan, norm, stream=None):
    c = Call(plan.device)
    c.run(gswa.lib().adamw_norm, stream, plan.c_ref, c.flat("norm", norm, torch.float32, 1))


def adamw_step(plan, step, lr, lr_scale=None, norm=None, max_norm=0.0, stream=None):
    c = Call(plan.device)
    c.run(gswa.lib().adamw_step, stream, plan.c_ref, c.flat("step", step, torch.int64, 1), lr,
          c.flat("lr_scale", lr_scale, torch.float32, 1), c.flat("norm", norm, torch.float32, 1), max_norm)


def adamw_unpack(plan, m_out, v_out, stream=None):
    c = Call(plan.device)
    c.run(gswa.lib().adamw_unpack, stream, plan.c_ref, c.flat("m_out", m_out, torch.bfloat16, plan.elements),
          c.flat("v_out", v_out, torch.bfloat16, plan.elements))
