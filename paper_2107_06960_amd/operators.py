"""The operators of a reader (include/mafat_reader.h): a decoder whose tokens, of many requests at once, read the feature
maps that a ``mafat.Network`` leaves on the device.

``mafat_add_rms_norm``, ``mafat_linear`` and ``mafat_cross_attention`` keep the C names and only marshal arguments
(device pointers and sizes).  ``add_rms_norm``, ``linear8`` and ``cross_attention`` take torch tensors on the GPU, check
them, allocate what they return and run on the current stream of the tensors' device.  There is no fallback: every step
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
EXPORTS = ("mafat_add_rms_norm", "mafat_linear_workspace", "mafat_linear", "mafat_cross_workspace",
           "mafat_cross_attention")


class mafat_adapters(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("rank", ctypes.c_int32), ("a", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("factor", ctypes.c_void_p), ("of_row", ctypes.c_void_p)]


class mafat_cross(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("frames", ctypes.c_int32), ("rows", ctypes.c_int64), ("positions", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
                    "q_row", "q_head", "k_frame", "k_pos", "k_head", "v_frame", "v_pos", "v_head", "y_row", "y_head",
                    "mask_row")] + [("mask_by_row", ctypes.c_int32)]


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
        crp = ctypes.POINTER(mafat_cross)
        L.mafat_cross_workspace.argtypes = [crp, ctypes.POINTER(sz)]
        L.mafat_cross_attention.argtypes = [crp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
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


def mafat_cross_workspace(c):
    """Bytes of workspace of a mafat_cross."""
    n = ctypes.c_size_t()
    M._check("mafat_cross_workspace", lib().mafat_cross_workspace(ctypes.byref(c), ctypes.byref(n)))
    return n.value


def mafat_cross_attention(c, q, k, v, q_offsets, k_lengths, mask, y, lse, workspace, ws_bytes, stream):
    """c: a mafat_cross; device pointers (int or None), stream: hipStream_t (int)."""
    M._check("mafat_cross_attention",
             lib().mafat_cross_attention(ctypes.byref(c), q, k, v, q_offsets, k_lengths, mask, y, lse, workspace, ws_bytes,
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


def cross_attention(q, k, v, q_offsets=None, k_lengths=None, key_mask=None, row_mask=None, scale=None, lse=False):
    """(y, lse): attention of query rows to the positions of the frames they are about, y in q's type.

    q: [rows, q_heads, d], the rows of all requests about frame 0, then those about frame 1, ...; k, v: [frames, positions,
    kv_heads, d] (e.g. the halves of a network's output channels; strides are free but for d's), all float32 or all
    bfloat16; q_heads a multiple of kv_heads, d up to 256.  q_offsets: int32 [frames + 1], frame f's rows are q_offsets[f]
    to q_offsets[f + 1] (None: rows / frames each; rows that no frame has come back undefined).  k_lengths: int32
    [frames], the valid positions of each (None: all).  key_mask: bool [frames, positions] or row_mask: bool [rows,
    positions], true where a position may be read.  scale: of q . k (None: 1 / sqrt(d)).  lse=True: the logarithm of each
    row's sum of exponentials, float32 [rows, q_heads], -inf for rows without any position (their y is 0); else None.
    """
    _need(q.is_cuda and q.dim() == 3 and q.dtype in (torch.float32, torch.bfloat16),
          "q must be a float32 or bfloat16 tensor [rows, heads, d] on the GPU")
    rows, hq, d = q.shape
    dev = q.device
    _need(k.dim() == 4 and k.shape == v.shape and k.shape[3] == d and k.dtype == q.dtype and v.dtype == q.dtype and
          k.device == dev and v.device == dev, f"k and v must be {q.dtype} tensors [frames, positions, heads, {d}] on {dev}")
    frames, positions, hkv, _ = k.shape
    _need(frames > 0 and hkv > 0 and hq > 0 and d > 0 and hq % hkv == 0,
          "there must be frames and heads, q's heads a multiple of k's")
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _need(d == 1 or t.stride(-1) == 1, f"{name} must have contiguous values of a head")
    _vector(q_offsets, frames + 1, torch.int32, dev, "q_offsets")
    _vector(k_lengths, frames, torch.int32, dev, "k_lengths")
    _need(key_mask is None or row_mask is None, "key_mask and row_mask exclude each other")
    mask, by_row, m_row = (key_mask, 0, 0) if row_mask is None else (row_mask, 1, 0)
    if mask is not None:
        n = rows if by_row else frames
        _need(mask.dtype == torch.bool and mask.shape == (n, positions) and mask.device == dev,
              f"the mask must be a bool tensor of shape {(n, positions)} on {dev}")
        m_row = _row_stride(mask, "the mask") if positions else 0
    y = torch.empty((rows, hq, d), dtype=q.dtype, device=dev)
    got = torch.empty((rows, hq), dtype=torch.float32, device=dev) if lse else None

    def of(t, i):  # an axis of one entry, or of a tensor without entries, may have any stride
        return t.stride(i) if t.shape[i] > 1 and t.numel() else max(t.stride(i), d)

    c = mafat_cross(_CODES[q.dtype], frames, rows, positions, hq, hkv, d, 1 / math.sqrt(d) if scale is None else scale,
                    of(q, 0), of(q, 1), of(k, 0), of(k, 1), of(k, 2), of(v, 0), of(v, 1), of(v, 2), hq * d, d, m_row, by_row)
    ref = ctypes.byref(c)
    need = ctypes.c_size_t()
    fn = (_ready or lib()).mafat_cross_workspace
    M._check("mafat_cross_workspace", fn(ref, ctypes.byref(need)))
    ws = torch.empty(need.value, dtype=torch.uint8, device=dev) if need.value else None
    _call("mafat_cross_attention", dev, ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(q_offsets), _ptr(k_lengths),
          _ptr(mask), y.data_ptr(), _ptr(got), _ptr(ws), need.value)
    return y, got
