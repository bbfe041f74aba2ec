"""The operators of a reader (include/mafat_reader.h): a decoder whose tokens, of many requests at once, read the feature
maps that a ``mafat.Network`` leaves on the device.

``mafat_add_rms_norm`` keeps the C name and only marshals arguments (device pointers and sizes).
``add_rms_norm`` takes torch tensors on the GPU, checks them,
allocates what it returns and runs on the current stream of the tensors' device.  There is no fallback: every step
runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import mafat as M

MAFAT_F8 = 2
F8 = torch.float8_e4m3fn
_CODES = {torch.float32: M.MAFAT_F32, torch.bfloat16: M.MAFAT_BF16, F8: MAFAT_F8}
_NAMES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": F8}

# Every symbol include/mafat_reader.h declares.
EXPORTS = ("mafat_add_rms_norm",)

_ready = None


def lib():
    """libmafat.so with the argument types of the reader's operators."""
    global _ready
    if _ready is None:
        L = M.lib()
        i32, i64, vp, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
        L.mafat_add_rms_norm.argtypes = [i64, i64, i32, vp, i64, vp, i64, vp, f32, vp, i64, i32, vp, i64, vp, vp]
        _ready = L
    return _ready


def _raw_stream(device):
    """The current stream of `device`, as M._stream_handle gives it for the current one."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None:
        return raw(device.index)
    return torch.cuda.current_stream(device).cuda_stream


class _On:
    """Makes `device` the current one for a call, if it is not."""

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _call(name, device, *args):
    """One C call on the current stream of `device`, its last argument."""
    fn = getattr(_ready or lib(), name)
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, _raw_stream(device))
    else:
        with _On(device):
            rc = fn(*args, _raw_stream(device))
    if rc:
        M._check(name, rc)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _vector(t, n, dtype, device, name):
    """An optional contiguous vector of n values."""
    if t is not None:
        _need(t.dtype == dtype and t.dim() == 1 and t.shape[0] == n and t.is_contiguous() and t.device == device,
              f"{name} must be a contiguous {dtype} vector of {n} values on {device}")


def _matrix(t, shape, dtype, device, name):
    """A matrix of contiguous rows; its row stride."""
    _need(t.dtype == dtype and t.shape == shape and t.device == device,
          f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return _row_stride(t, name)


def _row_stride(t, name):
    """Elements between the rows of a matrix whose rows are contiguous and apart (a single one counts as such)."""
    rows, cols = t.shape
    if rows <= 1:
        s = cols
    else:
        s = t.stride(0)
    _need((cols == 1 or t.stride(1) == 1) and s >= cols, f"{name} must have contiguous rows that do not overlap")
    return s


# ------------------------------------------------------------------ C names

def mafat_add_rms_norm(rows, cols, dtype, x, x_stride, residual, residual_stride, gain, eps, total, sum_stride, out_dtype,
                       y, y_stride, y_scale, stream):
    """Device pointers (int or None), strides in elements, dtype codes, stream: hipStream_t (int)."""
    M._check("mafat_add_rms_norm",
             lib().mafat_add_rms_norm(rows, cols, dtype, x, x_stride, residual, residual_stride, gain, eps, total,
                                      sum_stride, out_dtype, y, y_stride, y_scale, stream))


# ------------------------------------------------------------------ on tensors

def add_rms_norm(x, gain=None, residual=None, eps=1e-6, out="f8"):
    """(h, y, scale): h = x + residual in x's type (None without a residual), y = h / sqrt(mean(h^2) + eps) * gain.

    x, residual: [rows, cols], float32 or bfloat16, contiguous rows of any stride.  gain: float32 [cols] or None (ones).
    out: "f8" (e4m3 values with a float32 scale per row: y times scale is the norm), "bf16" or "f32" (scale is None).
    """
    _need(x.is_cuda and x.dim() == 2 and x.dtype in (torch.float32, torch.bfloat16),
          "x must be a float32 or bfloat16 matrix on the GPU")
    rows, cols = x.shape
    _need(cols > 0, "x has no columns")
    dev, to = x.device, _NAMES.get(out)
    _need(to is not None, f"out must be one of {sorted(_NAMES)}, not {out!r}")
    _vector(gain, cols, torch.float32, dev, "gain")
    h = None
    r_stride = cols
    if residual is not None:
        r_stride = _matrix(residual, x.shape, x.dtype, dev, "residual")
        h = torch.empty((rows, cols), dtype=x.dtype, device=dev)
    y = torch.empty((rows, cols), dtype=to, device=dev)
    scale = torch.empty(rows, dtype=torch.float32, device=dev) if to is F8 else None
    _call("mafat_add_rms_norm", dev, rows, cols, _CODES[x.dtype], x.data_ptr(), _row_stride(x, "x"), _ptr(residual),
          r_stride, _ptr(gain), eps, _ptr(h), cols, _CODES[to], y.data_ptr(), cols, _ptr(scale))
    return h, y, scale
