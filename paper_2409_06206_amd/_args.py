"""What the bindings of lnorm.h, relpos.h and adamw.h check about the tensors they are given, and the call itself.

A tensor of the wrong type, size or layout would be read out of its bounds by a kernel; raw addresses (integers) are the
caller's own.  Work goes to the device the tensors lie on and, where no stream is named, to that device's current stream.
"""
from .gswa import GSWA_BF16, GSWA_F32, _check

DTYPES = {"f32": GSWA_F32, "bf16": GSWA_BF16}


class Call:
    """One call: collects the device of its tensors."""

    def __init__(self):
        self.device = None

    def _seen(self, name, t, dtype):
        if not t.is_cuda:
            raise ValueError(f"{name} must lie on a GPU")
        if self.device is None:
            self.device = t.device
        elif t.device != self.device:
            raise ValueError(f"{name} lies on {t.device}, the tensors before it on {self.device}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, not {t.dtype}")

    def flat(self, name, t, dtype, numel):
        """Address of a contiguous tensor of at least `numel` elements."""
        if t is None or isinstance(t, int):
            return t
        self._seen(name, t, dtype)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.numel() < numel:
            raise ValueError(f"{name} has {t.numel()} elements, {numel} are needed")
        return t.data_ptr()

    def rows(self, name, t, dtype, rows, length, stride):
        """Address of `rows` rows of `length` elements, `stride` apart: contiguous in any shape, or 2-D."""
        if t is None or isinstance(t, int):
            return t
        self._seen(name, t, dtype)
        if t.is_contiguous() and (stride == length or rows == 1):
            if t.numel() != rows * length or t.shape[-1] != length:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, {rows} rows of {length} are needed")
        elif t.dim() != 2 or tuple(t.shape) != (rows, length) or (length > 1 and t.stride(1) != 1) or \
                (rows > 1 and t.stride(0) != stride):
            raise ValueError(f"{name} must be {rows} rows of {length} elements, {stride} apart; it has shape {tuple(t.shape)} "
                             f"and strides {t.stride()}")
        return t.data_ptr()

    def run(self, fn, stream, *args):
        """fn(*args, stream) on the tensors' device."""
        if self.device is None:       # raw addresses only
            if stream is None:
                import torch
                stream = torch.cuda.current_stream()
            _check(fn(*args, getattr(stream, "cuda_stream", stream)))
            return
        import torch
        at = getattr(stream, "device", None)
        if at is not None and at != self.device:
            raise ValueError(f"the stream belongs to {at}, the tensors lie on {self.device}")
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        handle = getattr(stream, "cuda_stream", stream)
        if torch.cuda.current_device() == self.device.index:
            _check(fn(*args, handle))
        else:
            with torch.cuda.device(self.device):
                _check(fn(*args, handle))


def torch_dtype(code):
    import torch
    return torch.float32 if code == GSWA_F32 else torch.bfloat16
