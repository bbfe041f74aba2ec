"""The operators of a reader (include/mafat_reader.h): a decoder whose tokens, of many requests at once, read the feature
maps that a ``mafat.Network`` leaves on the device.

``mafat_add_rms_norm``, ``mafat_linear``, ``mafat_cross_attention``, ``mafat_rotary``, ``mafat_decay_attention`` and
``mafat_block_norm`` keep the C names and only marshal arguments (device pointers and sizes).  ``add_rms_norm``, ``linear8``,
``cross_attention``, ``rotary``, ``decay_attention`` and ``block_norm`` take torch tensors on the GPU, check them, allocate
what they return and run on the current stream of the tensors' device.  There is no fallback: every step
runs in the library's HIP kernels.  They are forward only: a tensor that requires a gradient is refused while gradients are
recorded (call under torch.no_grad(), or pass it detached), and so is one with a tangent of forward-mode differentiation.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch
from torch.autograd import forward_ad as _forward

from . import mafat as M

MAFAT_F8 = 2
F8 = torch.float8_e4m3fn
_CODES = {torch.float32: M.MAFAT_F32, torch.bfloat16: M.MAFAT_BF16, F8: MAFAT_F8}
_NAMES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": F8}

# Every symbol include/mafat_reader.h declares.
EXPORTS = ("mafat_add_rms_norm", "mafat_linear_workspace", "mafat_linear", "mafat_cross_workspace",
           "mafat_cross_attention", "mafat_rotary", "mafat_block_norm", "mafat_decay_workspace", "mafat_decay_attention")


class mafat_adapters(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("rank", ctypes.c_int32), ("a", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("factor", ctypes.c_void_p), ("of_row", ctypes.c_void_p)]


class mafat_cross(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("frames", ctypes.c_int32), ("rows", ctypes.c_int64), ("positions", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
                    "q_row", "q_head", "k_frame", "k_pos", "k_head", "v_frame", "v_pos", "v_head", "y_row", "y_head",
                    "mask_row")] + [("mask_by_row", ctypes.c_int32)]


class mafat_turns(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("axes", ctypes.c_int32), ("rows", ctypes.c_int64), ("q_heads", ctypes.c_int32),
                ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("pairs", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
                    "q_row", "q_head", "k_row", "k_head", "qy_row", "qy_head", "ky_row", "ky_head")]


class mafat_block(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("after", ctypes.c_int32), ("groups", ctypes.c_int32), ("gate_act", ctypes.c_int32), ("before", ctypes.c_int32),
                ("eps", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
                    "x_stride", "gate_stride", "residual_stride", "sum_stride", "y_stride")]


class mafat_decay(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("requests", ctypes.c_int32), ("rows", ctypes.c_int64), ("slots", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("key_dim", ctypes.c_int32),
                ("value_dim", ctypes.c_int32), ("scale", ctypes.c_float), ("decay_by_row", ctypes.c_int32)] + [
                    (n, ctypes.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "y_row", "y_head",
                                                  "decay_row", "state_slot")]


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
        L.mafat_rotary.argtypes = [ctypes.POINTER(mafat_turns), vp, vp, vp, vp, vp, vp, vp]
        L.mafat_block_norm.argtypes = [ctypes.POINTER(mafat_block), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        dcp = ctypes.POINTER(mafat_decay)
        L.mafat_decay_workspace.argtypes = [dcp, ctypes.POINTER(sz)]
        L.mafat_decay_attention.argtypes = [dcp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        _ready = L
    return _ready


# The host's time counts where a call takes a few microseconds on the GPU: the
# current device and stream are asked for without building objects where torch
# offers that, and texts are put together only for an error.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_recording = torch.is_grad_enabled
_changed = torch.autograd.graph.increment_version  # for tensors that are written in place, through their addresses
_DENSE = torch.contiguous_format  # (empty_like takes a third less time than empty)


def _call(name, index, *args):
    """One C call on the current stream of device `index`, the call's last argument."""
    fn = getattr(_ready or lib(), name)
    before = _current_device()
    if before == index:
        rc = fn(*args, _raw_stream(index))
    else:
        torch.cuda.set_device(index)
        try:
            rc = fn(*args, _raw_stream(index))
        finally:
            torch.cuda.set_device(before)
    if rc:
        M._check(name, rc)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _refuse(text):
    raise ValueError(text)


def _wants_grad(t):
    return t is not None and t.requires_grad


def _in_forward_mode():
    return getattr(_forward, "_current_level", 0) >= 0


def _no_tangents(*tensors):
    """Refuses tangents of forward mode, which `requires_grad` does not tell of."""
    for t in tensors:
        if isinstance(t, torch.Tensor) and _forward.unpack_dual(t).tangent is not None:
            _forward_only()


def _forward_only():
    """Refuses what would come back without its gradient and without a word."""
    _refuse("the operators are forward only: call them under torch.no_grad(), or on detached tensors")


def _vector(t, n, dtype, dev, name):
    """The address of an optional contiguous vector of n values."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != (n,) or t.device != dev or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} vector of {n} values on {dev}")
    return t.data_ptr()


def _row_stride(t, name):
    """Elements between the rows of a matrix whose rows are contiguous and apart (a single one counts as such)."""
    rows, cols = t.shape
    s, c = t.stride()
    if rows <= 1:
        s = cols
    if (c != 1 and cols != 1) or s < cols:
        _refuse(f"{name} must have contiguous rows that do not overlap")
    return s


def _matrix(t, shape, dtype, dev, name):
    """The row stride of a matrix."""
    if t.dtype is not dtype or t.shape != shape or t.device != dev:
        _refuse(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return _row_stride(t, name)


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


def mafat_rotary(c, positions, turns, q, k, qy, ky, stream):
    """c: a mafat_turns; device pointers (int or None), stream: hipStream_t (int)."""
    M._check("mafat_rotary", lib().mafat_rotary(ctypes.byref(c), positions, turns, q, k, qy, ky, stream))


def mafat_block_norm(c, x, after_gain, gate, scale, residual, total, before_gain, y, y_scale, stream):
    """c: a mafat_block; device pointers (int or None), stream: hipStream_t (int)."""
    M._check("mafat_block_norm", lib().mafat_block_norm(ctypes.byref(c), x, after_gain, gate, scale, residual, total,
                                                        before_gain, y, y_scale, stream))


def mafat_decay_workspace(c):
    """Bytes of workspace of a mafat_decay."""
    n = ctypes.c_size_t()
    M._check("mafat_decay_workspace", lib().mafat_decay_workspace(ctypes.byref(c), ctypes.byref(n)))
    return n.value


def mafat_decay_attention(c, q, k, v, log_decay, offsets, states, slots, y, workspace, ws_bytes, stream):
    """c: a mafat_decay; device pointers (int or None), stream: hipStream_t (int)."""
    M._check("mafat_decay_attention",
             lib().mafat_decay_attention(ctypes.byref(c), q, k, v, log_decay, offsets, states, slots, y, workspace, ws_bytes,
                                         stream))


# ------------------------------------------------------------------ on tensors

def add_rms_norm(x, gain=None, residual=None, eps=1e-6, out="f8"):
    """(h, y, scale): h = x + residual in x's type (None without a residual), y = h / sqrt(mean(h^2) + eps) * gain.

    x, residual: [rows, cols], float32 or bfloat16, contiguous rows of any stride.  gain: float32 [cols] or None (ones).
    out: "f8" (e4m3 values with a float32 scale per row: y times scale is the norm), "bf16" or "f32" (scale is None).
    """
    dt, to = x.dtype, _NAMES.get(out)
    if not x.is_cuda or x.dim() != 2 or (dt is not torch.bfloat16 and dt is not torch.float32):
        _refuse("x must be a float32 or bfloat16 matrix on the GPU")
    if _recording() and (x.requires_grad or _wants_grad(gain) or _wants_grad(residual)):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(x, gain, residual)
    if to is None:
        _refuse(f"out must be one of {sorted(_NAMES)}, not {out!r}")
    rows, cols = x.shape
    if cols < 1:
        _refuse("x has no columns")
    dev = x.device
    x_stride = _row_stride(x, "x")
    gain_at = _vector(gain, cols, torch.float32, dev, "gain")
    h = h_at = res_at = None
    r_stride = cols
    if residual is not None:
        r_stride = _matrix(residual, x.shape, dt, dev, "residual")
        h = torch.empty((rows, cols), dtype=dt, device=dev)
        h_at, res_at = h.data_ptr(), residual.data_ptr()
    y = torch.empty((rows, cols), dtype=to, device=dev)
    scale = scale_at = None
    if to is F8:
        scale = torch.empty(rows, dtype=torch.float32, device=dev)
        scale_at = scale.data_ptr()
    _call("mafat_add_rms_norm", dev.index, rows, cols, _CODES[dt], x.data_ptr(), x_stride, res_at, r_stride, gain_at, eps,
          h_at, cols, _CODES[to], y.data_ptr(), cols, scale_at)
    return h, y, scale


def linear8(x, x_scale, w, w_scale, bias=None, adapters=None, row_adapter=None):
    """y = (x * x_scale) (w * w_scale)^T + bias, plus each row's low-rank adapter, in bfloat16.

    x: e4m3 [rows, in] with x_scale float32 [rows] (what add_rms_norm gives); w: e4m3 [out, in] with w_scale float32
    [out]; bias: float32 [out] or None.  adapters: (a, b, factor) of `count` adapters, a bfloat16 [count, rank, in], b
    bfloat16 [count, out, rank], factor float32 [count] or None, with row_adapter int32 [rows]: row i gets
    factor[j] * (x_i a[j]^T) b[j]^T for j = row_adapter[i], nothing where that is outside [0, count).
    """
    if not x.is_cuda or x.dim() != 2 or w.dim() != 2 or x.dtype is not F8:
        _refuse("x and w must be float8_e4m3fn matrices on the GPU")
    if _recording() and (x.requires_grad or w.requires_grad or _wants_grad(x_scale) or _wants_grad(w_scale) or
                         _wants_grad(bias) or (adapters is not None and any(map(_wants_grad, adapters)))):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(x, w, x_scale, w_scale, bias, *(adapters or ()))
    rows, k = x.shape
    n, dev = w.shape[0], x.device
    if k < 1 or n < 1:
        _refuse("x and w must have columns and rows")
    x_stride, w_stride = _row_stride(x, "x"), _matrix(w, (n, k), F8, dev, "w")
    x_scale_at = _vector(x_scale, rows, torch.float32, dev, "x_scale")
    w_scale_at = _vector(w_scale, n, torch.float32, dev, "w_scale")
    bias_at = _vector(bias, n, torch.float32, dev, "bias")
    if (adapters is None) != (row_adapter is None):
        _refuse("adapters and row_adapter go together")
    y = torch.empty((rows, n), dtype=torch.bfloat16, device=dev)
    ad = ws = None
    ws_bytes = 0
    if adapters is not None:
        a, b, factor = adapters
        if a.dim() != 3 or a.shape[0] < 1 or a.shape[1] < 1:
            _refuse("adapters must not be empty")
        count, rank, _ = a.shape
        for t, shape, name in ((a, (count, rank, k), "a"), (b, (count, n, rank), "b")):
            if t.dtype is not torch.bfloat16 or t.shape != shape or t.device != dev or not t.is_contiguous():
                _refuse(f"adapters' {name} must be a contiguous bfloat16 tensor of shape {shape} on {dev}")
        factor_at = _vector(factor, count, torch.float32, dev, "adapters' factor")
        of_row = _vector(row_adapter, rows, torch.int32, dev, "row_adapter")
        ad = ctypes.byref(mafat_adapters(count, rank, a.data_ptr(), b.data_ptr(), factor_at, of_row))
        need = ctypes.c_size_t()
        M._check("mafat_linear_workspace", (_ready or lib()).mafat_linear_workspace(rows, k, n, ad, ctypes.byref(need)))
        ws_bytes = need.value
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    _call("mafat_linear", dev.index, rows, k, n, x.data_ptr(), x_stride, x_scale_at, w.data_ptr(), w_stride, w_scale_at,
          bias_at, ad, y.data_ptr(), n, _ptr(ws), ws_bytes)
    return y


def cross_attention(q, k, v, q_offsets=None, k_lengths=None, key_mask=None, row_mask=None, scale=None, lse=False):
    """(y, lse): attention of query rows to the positions of the frames they are about, y in q's type.

    q: [rows, q_heads, d], the rows of all requests about frame 0, then those about frame 1, ...; k, v: [frames, positions,
    kv_heads, d] (e.g. the halves of a network's output channels; strides are free but for d's), all float32 or all
    bfloat16; q_heads a multiple of kv_heads, d up to 256.  q_offsets: int32 [frames + 1], frame f's rows are q_offsets[f]
    to q_offsets[f + 1] (None: rows / frames each; rows that no frame has come back undefined).  k_lengths: int32
    [frames], the valid positions of each (None: all).  key_mask: bool [frames, positions] or row_mask: bool [rows,
    positions], true where a position may be read.  scale: of q . k, a number (a tensor of one value is read on the host
    at every call; None: 1 / sqrt(d)).  lse=True: the logarithm of each
    row's sum of exponentials, float32 [rows, q_heads], -inf for rows without any position (their y is 0); else None.
    """
    dt = q.dtype
    if not q.is_cuda or q.dim() != 3 or (dt is not torch.bfloat16 and dt is not torch.float32):
        _refuse("q must be a float32 or bfloat16 tensor [rows, heads, d] on the GPU")
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad or getattr(scale, "requires_grad", False)):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(q, k, v, scale)
    rows, hq, d = q.shape
    dev, shape = q.device, k.shape
    if k.dim() != 4 or shape != v.shape or shape[3] != d or k.dtype is not dt or v.dtype is not dt or k.device != dev or \
            v.device != dev:
        _refuse(f"k and v must be {dt} tensors [frames, positions, heads, {d}] on {dev}")
    frames, positions, hkv, _ = shape
    mask, by_row = (key_mask, 0) if row_mask is None else (row_mask, 1)
    m_row = 0
    if mask is not None:
        if key_mask is not None and row_mask is not None:
            _refuse("key_mask and row_mask exclude each other")
        if mask.dtype is not torch.bool or mask.shape != (rows if by_row else frames, positions) or mask.device != dev:
            _refuse(f"the mask must be a bool tensor of shape {(rows if by_row else frames, positions)} on {dev}")
        m_row = _row_stride(mask, "the mask") if positions else 0
    offsets_at = _vector(q_offsets, frames + 1, torch.int32, dev, "q_offsets")
    lengths_at = _vector(k_lengths, frames, torch.int32, dev, "k_lengths")
    if scale is not None:
        scale = float(scale)  # of a tensor its value now: the shapes below are kept by what they hold
    ref, need, _ = _cross_shape(dt, rows, hq, d, frames, positions, hkv, q.stride(), k.stride(), v.stride(), scale, m_row, by_row)
    y = torch.empty((rows, hq, d), dtype=dt, device=dev)
    got = torch.empty((rows, hq), dtype=torch.float32, device=dev) if lse else None
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call("mafat_cross_attention", dev.index, ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets_at, lengths_at, _ptr(mask),
          y.data_ptr(), _ptr(got), _ptr(ws), need)
    return y, got


@functools.lru_cache(maxsize=256)
def _cross_shape(dt, rows, hq, d, frames, positions, hkv, qs, ks, vs, scale, m_row, by_row):
    """(reference to the call's mafat_cross, bytes of workspace, the struct itself) for sizes and strides."""
    if not (frames > 0 and hkv > 0 and hq > 0 and d > 0 and hq % hkv == 0):
        _refuse("there must be frames and heads, q's heads a multiple of k's")
    if d > 1 and not qs[2] == ks[3] == vs[3] == 1:
        _refuse("q, k and v must have contiguous values of a head")

    def of(stride, n, entries):  # an axis of one entry, or of a tensor without entries, may have any stride
        return stride if n > 1 and entries else max(stride, d)

    some = frames * positions
    c = mafat_cross(_CODES[dt], frames, rows, positions, hq, hkv, d, 1 / math.sqrt(d) if scale is None else scale,
                    of(qs[0], rows, rows), of(qs[1], hq, rows), *(of(st[i], n, some) for st in (ks, vs) for i, n in (
                        (0, frames), (1, positions), (2, hkv))), hq * d, d, m_row, by_row)
    need = mafat_cross_workspace(c)
    return ctypes.byref(c), need, c


def rotary_turns(pairs, base=10000.0, stretch=1.0, trained=None, slow=1.0, fast=32.0, device="cuda"):
    """Turns per step of `pairs` pairs (what rotary takes): base^(-i / pairs) / (2 pi), float64 [pairs].

    stretch: by how much contexts are longer than trained ones; every frequency is divided by it.  With `trained`, the
    trained length, only frequencies that turn less than `slow` times within it are, those that turn more than `fast` times
    are kept, and in between the share goes linearly by the number of turns.
    """
    turns = base ** (-torch.arange(pairs, dtype=torch.float64, device=device) / max(pairs, 1)) / (2 * math.pi)
    if trained is None:
        return turns / stretch
    keep = ((turns * trained - slow) / (fast - slow)).clamp(0, 1)
    return turns * (keep + (1 - keep) / stretch)


def rotary(q, positions, turns, k=None, interleaved=False, magnitude=1.0, in_place=False):
    """(q', k'): q and k with the first pairs of every head turned by their row's position (k' is None without k).

    q: [rows, q_heads, d] and k: [rows, k_heads, d], float32 or bfloat16, of any row and head strides (e.g. parts of one
    projection's rows).  positions: int32 [rows] or [rows, axes].  turns: float64 [pairs] or [axes, pairs], turns per step
    (rotary_turns); pair i turns by 2 pi sum_a positions[:, a] turns[a, i].  A pair is values i and pairs + i, or, interleaved,
    2 i and 2 i + 1; values behind the pairs stay as they are.  magnitude: a factor of the turned values.  in_place: q and k
    are overwritten and returned.
    """
    dt = q.dtype
    if not q.is_cuda or q.dim() != 3 or (dt is not torch.bfloat16 and dt is not torch.float32):
        _refuse("q must be a float32 or bfloat16 tensor [rows, heads, d] on the GPU")
    if _recording() and (q.requires_grad or _wants_grad(k) or turns.requires_grad or getattr(magnitude, "requires_grad", False)):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(q, k, turns, magnitude)
    rows, hq, d = q.shape
    dev, hk, ks = q.device, 0, None
    if k is not None:
        if k.dim() != 3 or k.dtype is not dt or k.device != dev or k.shape[0] != rows or k.shape[2] != d or k.shape[1] < 1:
            _refuse(f"k must be a {dt} tensor [{rows}, heads, {d}] on {dev}")
        hk, ks = k.shape[1], k.stride()
    axes = positions.shape[1] if positions.dim() == 2 else 1
    if positions.dtype is not torch.int32 or positions.shape not in ((rows,), (rows, axes)) or positions.device != dev or \
            not positions.is_contiguous():
        _refuse(f"positions must be a contiguous int32 tensor [{rows}] or [{rows}, axes] on {dev}")
    pairs = turns.shape[-1] if turns.dim() else 0
    if turns.dtype is not torch.float64 or turns.shape not in ((axes, pairs), (pairs,) if axes == 1 else None) or \
            turns.device != dev or not turns.is_contiguous():
        _refuse(f"turns must be a contiguous float64 tensor [{axes}, pairs] on {dev}")
    ref, _ = _rotary_shape(dt, rows, hq, hk, d, axes, pairs, bool(interleaved), float(magnitude), q.stride(), ks, bool(in_place))
    if in_place:
        qy, ky = q, k
    else:
        qy = torch.empty_like(q, memory_format=_DENSE)
        ky = None if k is None else torch.empty_like(k, memory_format=_DENSE)
    _call("mafat_rotary", dev.index, ref, positions.data_ptr(), turns.data_ptr(), q.data_ptr(), _ptr(k), qy.data_ptr(), _ptr(ky))
    if in_place:
        _changed(q if k is None else (q, k))
    return qy, ky


def _outer(stride, n, entries, width):
    """The stride of an axis of n entries (one of a single entry, or of a tensor without entries, may have any)."""
    return stride if n > 1 and entries else max(stride, width)


@functools.lru_cache(maxsize=256)
def _rotary_shape(dt, rows, hq, hk, d, axes, pairs, interleaved, magnitude, qs, ks, in_place):
    """(reference to the call's mafat_turns, the struct itself) for sizes and strides."""
    if hq < 1 or d < 1:
        _refuse("q must have heads and values")
    if d > 1 and (qs[2] != 1 or (ks is not None and ks[2] != 1)):
        _refuse("q and k must have contiguous values of a head")
    q = _outer(qs[0], rows, rows, d), _outer(qs[1], hq, rows, d)
    k = (_outer(ks[0], rows, rows, d), _outer(ks[1], hk, rows, d)) if ks is not None else (d, d)
    out = (*q, *k) if in_place else (hq * d, d, max(hk, 1) * d, d)
    c = mafat_turns(_CODES[dt], axes, rows, hq, hk, d, pairs, interleaved, magnitude, *q, *k, *out)
    return ctypes.byref(c), c


def block_norm(x, after=True, after_gain=None, groups=1, gate=None, act="silu", scale=None, residual=None, before=True,
               before_gain=None, eps=1e-6, out="f8"):
    """(h, y, y_scale): a block's output x on its way into the residual stream and the next block.

        u = x / sqrt(mean(x^2) + eps) * after_gain      if after, the mean over each of `groups` equal parts of a row
        u = u * act(gate)                               with a gate; act: "silu" (gate * sigmoid(gate)) or "sigmoid"
        h = residual + scale * u
        y = h / sqrt(mean(h^2) + eps) * before_gain     if before

    x, gate, residual: [rows, cols], float32 or bfloat16 alike, contiguous rows of any stride.  after_gain, scale,
    before_gain: float32 [cols] or None (ones).  h comes back in x's type (None without a residual); y follows from h before
    that rounding.  out and y_scale as for add_rms_norm.
    """
    dt, to = x.dtype, _NAMES.get(out)
    if not x.is_cuda or x.dim() != 2 or (dt is not torch.bfloat16 and dt is not torch.float32):
        _refuse("x must be a float32 or bfloat16 matrix on the GPU")
    if _recording() and (x.requires_grad or _wants_grad(after_gain) or _wants_grad(gate) or _wants_grad(scale) or
                         _wants_grad(residual) or _wants_grad(before_gain)):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(x, after_gain, gate, scale, residual, before_gain)
    if to is None:
        _refuse(f"out must be one of {sorted(_NAMES)}, not {out!r}")
    if act != "silu" and act != "sigmoid":
        _refuse(f"act must be 'silu' or 'sigmoid', not {act!r}")
    rows, cols = shape = x.shape
    if cols < 1:
        _refuse("x has no columns")
    dev = x.device
    x_stride = _row_stride(x, "x")
    after_at = _vector(after_gain, cols, torch.float32, dev, "after_gain")
    before_at = _vector(before_gain, cols, torch.float32, dev, "before_gain")
    scale_at = _vector(scale, cols, torch.float32, dev, "scale")
    h = h_at = res_at = gate_at = y_scale = y_scale_at = None
    g_stride = r_stride = cols
    if gate is not None:
        g_stride = _matrix(gate, shape, dt, dev, "gate")
        gate_at = gate.data_ptr()
    if residual is not None:
        r_stride = _matrix(residual, shape, dt, dev, "residual")
        h = torch.empty_like(x, memory_format=_DENSE)
        h_at, res_at = h.data_ptr(), residual.data_ptr()
    y = torch.empty_like(x, dtype=to, memory_format=_DENSE)
    if to is F8:
        y_scale = torch.empty(rows, dtype=torch.float32, device=dev)
        y_scale_at = y_scale.data_ptr()
    # (of a tensor its value now: the shapes below are kept by what they hold)
    ref, _ = _block_shape(dt, to, rows, cols, bool(after), int(groups), act == "silu", bool(before), float(eps), x_stride, g_stride,
                          r_stride)
    _call("mafat_block_norm", dev.index, ref, x.data_ptr(), after_at, gate_at, scale_at, res_at, h_at, before_at, y.data_ptr(),
          y_scale_at)
    return h, y, y_scale


@functools.lru_cache(maxsize=256)
def _block_shape(dt, to, rows, cols, after, groups, silu, before, eps, x_stride, g_stride, r_stride):
    """(reference to the call's mafat_block, the struct itself)."""
    c = mafat_block(_CODES[dt], _CODES[to], rows, cols, after, groups, silu, before, eps, x_stride, g_stride, r_stride, cols, cols)
    return ctypes.byref(c), c


def decay_attention(q, k, v, log_decay, states=None, slots=None, offsets=None, scale=None):
    """y: linear attention among the tokens of each request, with a decay for each head; [rows, q_heads, dv] in q's type.

        S_t = exp(log_decay_t) S_(t-1) + k_t v_t^T,  y_t = scale * q_t S_t

    q: [rows, q_heads, dk], k: [rows, kv_heads, dk], v: [rows, kv_heads, dv], the tokens of request 0, then those of request
    1, ..., all float32 or all bfloat16, strides free but for the last; q_heads a multiple of kv_heads, dk and dv up to 256.
    log_decay: float32 [kv_heads] or [rows, kv_heads], at most 0 (above counts as 0).  states: float32 [slots, kv_heads, dk, dv],
    where each request's state is read from and, updated, kept in place (None: zeros, and nothing is kept); slots: int32
    [requests], each request's state (outside [0, slots): zeros, not kept; one that an earlier request has: y is NaN and
    the state is that request's), None: request i has state i.  offsets: int32 [requests + 1], request i's rows are offsets[i]
    to offsets[i + 1] (None: as many each; rows that no request has come back undefined).  The number of requests is that of
    offsets, of slots, of states, or 1.  scale: a number (None: 1 / sqrt(dk)).
    """
    dt = q.dtype
    if not q.is_cuda or q.dim() != 3 or (dt is not torch.bfloat16 and dt is not torch.float32):
        _refuse("q must be a float32 or bfloat16 tensor [rows, heads, d] on the GPU")
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad or log_decay.requires_grad or
                         _wants_grad(states) or getattr(scale, "requires_grad", False)):
        _forward_only()
    if _in_forward_mode():
        _no_tangents(q, k, v, log_decay, states, scale)
    rows, hq, dk = q.shape
    dev = q.device
    if k.dim() != 3 or k.dtype is not dt or k.device != dev or k.shape[0] != rows or k.shape[2] != dk:
        _refuse(f"k must be a {dt} tensor [{rows}, heads, {dk}] on {dev}")
    hkv = k.shape[1]
    if v.dim() != 3 or v.dtype is not dt or v.device != dev or v.shape[:2] != (rows, hkv):
        _refuse(f"v must be a {dt} tensor [{rows}, {hkv}, d] on {dev}")
    dv = v.shape[2]
    by_row = log_decay.dim() == 2
    if log_decay.dtype is not torch.float32 or log_decay.device != dev or log_decay.shape != ((rows, hkv) if by_row else (hkv,)):
        _refuse(f"log_decay must be a float32 tensor [{hkv}] or [{rows}, {hkv}] on {dev}")
    d_row = _row_stride(log_decay, "log_decay") if by_row else hkv
    if not by_row and hkv > 1 and log_decay.stride(0) != 1:
        _refuse("log_decay must be contiguous")
    pool, states_at, s_slot = 0, None, hkv * dk * dv
    if states is not None:
        if states.dtype is not torch.float32 or states.device != dev or states.dim() != 4 or states.shape[1:] != (hkv, dk, dv):
            _refuse(f"states must be a float32 tensor [slots, {hkv}, {dk}, {dv}] on {dev}")
        pool = states.shape[0]
        if pool and not states[0].is_contiguous():
            _refuse("states must be contiguous but for their first axis")
        states_at = states.data_ptr()
        s_slot = _outer(states.stride(0), pool, pool, s_slot)
    if offsets is not None:
        requests = offsets.numel() - 1
    elif slots is not None:
        requests = slots.numel()
    else:
        requests = pool if states is not None else 1
    if slots is not None and states is None:
        _refuse("slots need states")
    offsets_at = _vector(offsets, requests + 1, torch.int32, dev, "offsets")
    slots_at = _vector(slots, requests, torch.int32, dev, "slots")
    if scale is not None:
        scale = float(scale)  # of a tensor its value now: the shapes below are kept by what they hold
    ref, need, _ = _decay_shape(dt, requests, rows, pool, hq, hkv, dk, dv, scale, by_row, q.stride(), k.stride(), v.stride(), d_row,
                                s_slot)
    y = torch.empty_like(q, memory_format=_DENSE) if dv == dk else torch.empty((rows, hq, dv), dtype=dt, device=dev)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call("mafat_decay_attention", dev.index, ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), offsets_at,
          states_at, slots_at, y.data_ptr(), _ptr(ws), need)
    if states is not None:
        _changed(states)
    return y


@functools.lru_cache(maxsize=256)
def _decay_shape(dt, requests, rows, pool, hq, hkv, dk, dv, scale, by_row, qs, ks, vs, d_row, s_slot):
    """(reference to the call's mafat_decay, bytes of workspace, the struct itself) for sizes and strides."""
    if not (requests > 0 and hkv > 0 and hq > 0 and dk > 0 and dv > 0 and hq % hkv == 0):
        _refuse("there must be requests, heads and values, q's heads a multiple of k's")
    if (dk > 1 and not qs[2] == ks[2] == 1) or (dv > 1 and vs[2] != 1):
        _refuse("q, k and v must have contiguous values of a head")
    axes = [_outer(st[i], n, rows, d) for st, h, d in ((qs, hq, dk), (ks, hkv, dk), (vs, hkv, dv)) for i, n in ((0, rows), (1, h))]
    c = mafat_decay(_CODES[dt], requests, rows, pool, hq, hkv, dk, dv, 1 / math.sqrt(dk) if scale is None else scale, by_row, *axes,
                    hq * dv, dv, d_row, s_slot)
    need = mafat_decay_workspace(c)
    return ctypes.byref(c), need, c
