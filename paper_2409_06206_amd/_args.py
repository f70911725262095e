"""What the bindings of lnorm.h, relpos.h and adamw.h check about the tensors they are given, and the call itself.

A tensor of the wrong type, size or layout would be read out of its bounds by a kernel; raw addresses (integers) are the
caller's own.  Work goes to the device the tensors lie on and, where no stream is named, to that device's current stream.
"""
import ctypes
import operator

import torch

from .gswa import GSWA_BF16, GSWA_F32, GSWA_OK, _check

DTYPES = {"f32": GSWA_F32, "bf16": GSWA_BF16}
TORCH_DTYPES = {GSWA_F32: torch.float32, GSWA_BF16: torch.bfloat16}
# (the handle alone: torch.cuda.current_stream() builds a stream object around it, 1.8 us of a call of 5)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def torch_dtype(code):
    return TORCH_DTYPES.get(code, torch.bfloat16)   # (a code that is none is refused by the library)


class Whole:
    """The whole numbers of a structure: ctypes cuts off what a field cannot hold, and what is left may be another valid number."""

    def __init__(self, kind):
        self.names = tuple(n for n, t in kind._fields_ if t in (ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_uint64))
        self.of = operator.attrgetter(*self.names)

    def held(self, made, *given):
        """`made`, whose whole numbers have to be the `given` ones."""
        if self.of(made) != given:
            raise ValueError("; ".join(f"{n} cannot hold {v}" for n, v in zip(self.names, given) if getattr(made, n) != v))
        return made


class Specs(dict):
    """What the calls of a descriptor need of their tensors, by the descriptor's bytes: found once, since a small call takes no longer than finding it."""

    MOST = 1024

    def __init__(self, find):
        super().__init__()
        self.find = find

    def of(self, desc):
        key = bytes(desc)
        spec = self.get(key)
        if spec is None:
            if len(self) >= self.MOST:
                self.clear()
            spec = self[key] = self.find(desc)
        return spec


def row_spec(rows, length, stride):
    return (rows, length), (stride, 1)


class Call:
    """One call: `device` is the index of the device its tensors lie on, None before the first."""

    __slots__ = ("device",)

    def __init__(self, device=None):
        self.device = device

    def _place(self, name, t, dtype):
        at = t.get_device()
        if at < 0:
            raise ValueError(f"{name} must lie on a GPU")
        if self.device is None:
            self.device = at
        elif at != self.device:
            raise ValueError(f"{name} lies on device {at}, the tensors before it on device {self.device}")
        if t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype}, not {t.dtype}")

    def flat(self, name, t, dtype, numel):
        """Address of a contiguous tensor of at least `numel` elements."""
        if t is None or t.__class__ is int:
            return t
        if t.get_device() != self.device or t.dtype is not dtype:
            self._place(name, t, dtype)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.numel() < numel:
            raise ValueError(f"{name} has {t.numel()} elements, {numel} are needed")
        return t.data_ptr()

    def rows(self, name, t, dtype, spec):
        """Address of rows as row_spec names them: contiguous in any shape, or 2-D."""
        if t is None or t.__class__ is int:
            return t
        if t.get_device() != self.device or t.dtype is not dtype:
            self._place(name, t, dtype)
        if t.shape != spec[0] or t.stride() != spec[1]:
            self._other_rows(name, t, spec)
        return t.data_ptr()

    @staticmethod
    def _other_rows(name, t, spec):
        (rows, length), (stride, _) = spec
        if t.is_contiguous() and (stride == length or rows == 1):
            if t.numel() != rows * length or t.shape[-1] != length:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, {rows} rows of {length} are needed")
        elif t.dim() != 2 or t.shape != (rows, length) or (length > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) != stride):
            raise ValueError(f"{name} must be {rows} rows of {length} elements, {stride} apart; it has shape {tuple(t.shape)} "
                             f"and strides {t.stride()}")

    def run(self, fn, stream, *args):
        """fn(*args, stream) on the tensors' device."""
        if self.device is None:       # raw addresses only
            if stream is None:
                stream = torch.cuda.current_stream()
            _check(fn(*args, getattr(stream, "cuda_stream", stream)))
            return
        if stream is None:
            stream = _raw_stream(self.device)
        elif not isinstance(stream, int):
            if stream.device_index != self.device:
                raise ValueError(f"the stream belongs to device {stream.device_index}, the tensors lie on device {self.device}")
            stream = stream.cuda_stream
        if _current_device() == self.device:
            status = fn(*args, stream)
            if status != GSWA_OK:
                _check(status)
        else:
            with torch.cuda.device(self.device):
                _check(fn(*args, stream))
