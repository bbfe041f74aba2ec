"""The operators of a reader (include/mafat_reader.h): a decoder whose tokens, of many requests at once, read the feature
maps that a ``mafat.Network`` leaves on the device.

``mafat_add_rms_norm`` and ``mafat_linear`` keep the C names and only marshal arguments (device pointers and sizes).
``add_rms_norm`` and ``linear8`` take torch tensors on the GPU, check them, allocate what they return and run on the
current stream of the tensors' device.  There is no fallback: every step runs in the library's HIP kernels.
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
EXPORTS = ("mafat_add_rms_norm", "mafat_linear_workspace", "mafat_linear")


class mafat_adapters(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("rank", ctypes.c_int32), ("a", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("factor", ctypes.c_void_p), ("of_row", ctypes.c_void_p)]


_ready = None


def lib():
    """libmafat.so with the argument types of the reader's operators."""
    global _ready
    if _ready is None:
        L = M.lib()
        i32, i64, vp, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
        L.mafat_add_rms_norm.argtypes = [i64, i64, i32, vp, i64, vp, i64, vp, f32, vp, i64, i32, vp, i64, vp, vp]
        adp, sz = ctypes.POINTER(mafat_adapters), ctypes.c_size_t
        L.mafat_linear_workspace.argtypes = [i64, i64, i64, adp, ctypes.POINTER(sz)]
        L.mafat_linear.argtypes = [i64, i64, i64, vp, i64, vp, vp, i64, vp, vp, adp, vp, i64, vp, sz, vp]
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


def mafat_linear_workspace(rows, in_cols, out_cols, adapters=None):
    """Bytes of workspace; adapters: a mafat_adapters or None."""
    n = ctypes.c_size_t()
    M._check("mafat_linear_workspace",
             lib().mafat_linear_workspace(rows, in_cols, out_cols, None if adapters is None else ctypes.byref(adapters),
                                          ctypes.byref(n)))
    return n.value


def mafat_linear(rows, in_cols, out_cols, x, x_stride, x_scale, w, w_stride, w_scale, bias, adapters, y, y_stride,
                 workspace, ws_bytes, stream):
    """Device pointers (int or None), adapters: a mafat_adapters or None, stream: hipStream_t (int)."""
    M._check("mafat_linear",
             lib().mafat_linear(rows, in_cols, out_cols, x, x_stride, x_scale, w, w_stride, w_scale, bias,
                                None if adapters is None else ctypes.byref(adapters), y, y_stride, workspace, ws_bytes,
                                stream))


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


def linear8(x, x_scale, w, w_scale, bias=None, adapters=None, row_adapter=None):
    """y = (x * x_scale) (w * w_scale)^T + bias, plus each row's low-rank adapter, in bfloat16.

    x: e4m3 [rows, in] with x_scale float32 [rows] (what add_rms_norm gives); w: e4m3 [out, in] with w_scale float32
    [out]; bias: float32 [out] or None.  adapters: (a, b, factor) of `count` adapters, a bfloat16 [count, rank, in], b
    bfloat16 [count, out, rank], factor float32 [count] or None, with row_adapter int32 [rows]: row i gets
    factor[j] * (x_i a[j]^T) b[j]^T for j = row_adapter[i], nothing where that is outside [0, count).
    """
    _need(x.is_cuda and x.dim() == 2 and w.dim() == 2 and x.dtype is F8, "x and w must be float8_e4m3fn matrices on the GPU")
    rows, k = x.shape
    n, dev = w.shape[0], x.device
    _need(k > 0 and n > 0, "x and w must have columns and rows")
    w_stride = _matrix(w, (n, k), F8, dev, "w")
    _vector(x_scale, rows, torch.float32, dev, "x_scale")
    _vector(w_scale, n, torch.float32, dev, "w_scale")
    _vector(bias, n, torch.float32, dev, "bias")
    _need((adapters is None) == (row_adapter is None), "adapters and row_adapter go together")
    y = torch.empty((rows, n), dtype=torch.bfloat16, device=dev)
    ad = ws = None
    ws_bytes = 0
    if adapters is not None:
        a, b, factor = adapters
        count, rank = a.shape[0], a.shape[1]
        _need(count > 0 and rank > 0, "adapters must not be empty")
        for t, shape, name in ((a, (count, rank, k), "adapters' a"), (b, (count, n, rank), "adapters' b")):
            _need(t.dtype == torch.bfloat16 and t.shape == shape and t.is_contiguous() and t.device == dev,
                  f"{name} must be a contiguous bfloat16 tensor of shape {shape} on {dev}")
        _vector(factor, count, torch.float32, dev, "adapters' factor")
        _vector(row_adapter, rows, torch.int32, dev, "row_adapter")
        ad = ctypes.byref(mafat_adapters(count, rank, a.data_ptr(), b.data_ptr(), _ptr(factor), row_adapter.data_ptr()))
        need = ctypes.c_size_t()
        M._check("mafat_linear_workspace", lib().mafat_linear_workspace(rows, k, n, ad, ctypes.byref(need)))
        ws_bytes = need.value
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    _call("mafat_linear", dev, rows, k, n, x.data_ptr(), _row_stride(x, "x"), _ptr(x_scale), w.data_ptr(), w_stride,
          _ptr(w_scale), _ptr(bias), ad, y.data_ptr(), n, _ptr(ws), ws_bytes)
    return y
