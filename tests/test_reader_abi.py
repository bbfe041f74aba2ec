"""CPU tests of the reader's C entries (include/mafat_reader.h): every declared symbol is exported, and each refusal comes
back as its status before any HIP call (pointers below are never followed)."""
import os
import re

import pytest

from paper_2107_06960_amd import mafat as M
from paper_2107_06960_amd import operators as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED = M.MAFAT_EINVAL, M.MAFAT_EUNSUPPORTED
F32, BF16, F8 = M.MAFAT_F32, M.MAFAT_BF16, O.MAFAT_F8
A, B, C, D, E = (k << 32 for k in range(1, 6))  # device addresses far apart


def test_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "mafat_reader.h")).read()
    declared = set(re.findall(r"\bint (mafat_[a-z_0-9]+)\s*\(", hdr))
    assert declared == set(O.EXPORTS)
    for name in declared:
        assert hasattr(O.lib(), name), name


NORM = dict(rows=4, cols=64, dtype=BF16, x=A, x_stride=64, residual=B, residual_stride=64, gain=C, eps=1e-6, sum=D,
            sum_stride=64, out_dtype=F8, y=E, y_stride=64, y_scale=E + (1 << 31), stream=None)


@pytest.mark.parametrize("change, status", [
    (dict(dtype=F8), EUNSUPPORTED), (dict(dtype=7), EUNSUPPORTED), (dict(out_dtype=3), EUNSUPPORTED),
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(rows=1 << 31), EUNSUPPORTED),
    (dict(cols=1 << 31, x_stride=1 << 31, residual_stride=1 << 31, sum_stride=1 << 31, y_stride=1 << 31), EUNSUPPORTED),
    (dict(eps=-1e-6), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL),
    (dict(residual=None), EINVAL), (dict(sum=None), EINVAL), (dict(y_scale=None), EINVAL), (dict(out_dtype=BF16), EINVAL),
    (dict(x_stride=63), EINVAL), (dict(residual_stride=0), EINVAL), (dict(sum_stride=-64), EINVAL), (dict(y_stride=1), EINVAL),
    (dict(x_stride=1 << 31), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(x=A + 1), EINVAL), (dict(gain=C + 2), EINVAL),
    (dict(y_scale=E + (1 << 31) + 2), EINVAL), (dict(dtype=F32, x=A + 2), EINVAL),
    # overlaps: y on x, on the sum, the sum shifted on x, the scales in y
    (dict(y=A), EINVAL), (dict(y=D + 256), EINVAL), (dict(sum=A + 2), EINVAL), (dict(sum=B, sum_stride=128), EINVAL),
    (dict(y_scale=E + 64), EINVAL),
    # side by side in one buffer's rows, but one column too near
    (dict(y=A + 193, x_stride=128, y_stride=256, cols=64), EINVAL),
])
def test_norm_refusals(change, status):
    rc = O.lib().mafat_add_rms_norm(*dict(NORM, **change).values())
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_norm_of_no_rows_is_valid():
    assert O.lib().mafat_add_rms_norm(*dict(NORM, rows=0).values()) == 0


def _adapters(**change):
    return O.mafat_adapters(**dict(dict(count=3, rank=8, a=C, b=C + (1 << 24), factor=C + (1 << 25), of_row=C + (1 << 26)),
                                   **change))


LINEAR = dict(rows=20, in_cols=64, out_cols=48, x=A, x_stride=64, x_scale=A + (1 << 30), w=B, w_stride=64,
              w_scale=B + (1 << 30), bias=B + (1 << 31), adapters=None, y=D, y_stride=48, workspace=E, ws_bytes=1024,
              stream=None)


@pytest.mark.parametrize("change, status", [
    (dict(rows=-1), EINVAL), (dict(in_cols=0), EINVAL), (dict(out_cols=0), EINVAL), (dict(rows=1 << 31), EUNSUPPORTED),
    (dict(in_cols=1 << 22, x_stride=1 << 22, w_stride=1 << 22), EUNSUPPORTED), (dict(out_cols=1 << 22), EUNSUPPORTED),
    (dict(x_stride=63), EINVAL), (dict(w_stride=0), EINVAL), (dict(y_stride=47), EINVAL),
    (dict(x_stride=1 << 22), EUNSUPPORTED), (dict(w_stride=1 << 22), EUNSUPPORTED), (dict(y_stride=1 << 31), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(x_scale=None), EINVAL), (dict(w_scale=None), EINVAL),
    (dict(y=None), EINVAL), (dict(y=D + 1), EINVAL), (dict(x_scale=A + (1 << 30) + 2), EINVAL),
    (dict(bias=B + (1 << 31) + 1), EINVAL),
    (dict(y=A), EINVAL), (dict(y=B + 64 * 47), EINVAL), (dict(y=B + (1 << 31)), EINVAL),
    (dict(adapters=_adapters(count=0)), EINVAL), (dict(adapters=_adapters(rank=0)), EINVAL),
    (dict(adapters=_adapters(rank=129)), EUNSUPPORTED), (dict(adapters=_adapters(a=None)), EINVAL),
    (dict(adapters=_adapters(b=None)), EINVAL), (dict(adapters=_adapters(of_row=None)), EINVAL),
    (dict(adapters=_adapters(of_row=C + 2)), EINVAL), (dict(adapters=_adapters(a=C + 1)), EINVAL),
    (dict(adapters=_adapters(), ws_bytes=639), M.MAFAT_EWORKSPACE), (dict(adapters=_adapters(), workspace=None), EINVAL),
    (dict(adapters=_adapters(), workspace=E + 128), EINVAL), (dict(adapters=_adapters(), workspace=D), EINVAL),
    (dict(adapters=_adapters(), workspace=A), EINVAL), (dict(adapters=_adapters(), y=C), EINVAL),
])
def test_linear_refusals(change, status):
    rc = O.lib().mafat_linear(*dict(LINEAR, **change).values())
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_linear_workspace_and_no_rows():
    assert O.mafat_linear_workspace(20, 64, 48) == 0
    assert O.mafat_linear_workspace(20, 64, 48, _adapters()) >= 20 * 8 * 4
    assert O.lib().mafat_linear_workspace(20, 64, 48, None, None) == EINVAL
    assert O.lib().mafat_linear(*dict(LINEAR, rows=0).values()) == 0
    assert O.lib().mafat_linear(*dict(LINEAR, rows=0, adapters=_adapters(), ws_bytes=0, workspace=None).values()) == 0


CROSS = dict(dtype=BF16, frames=2, rows=6, positions=40, q_heads=4, kv_heads=2, head_dim=64, scale=0.125, q_row=256, q_head=64,
             k_frame=40 * 256, k_pos=256, k_head=64, v_frame=40 * 256, v_pos=256, v_head=64, y_row=256, y_head=64, mask_row=40,
             mask_by_row=0)
CALL = dict(q=A, k=B, v=B + 256, q_offsets=C, k_lengths=C + 4096, mask=C + 8192, y=D, lse=D + (1 << 30), workspace=E,
            ws_bytes=1 << 30, stream=None)


def _cross(shape, call):
    import ctypes
    return O.lib().mafat_cross_attention(ctypes.byref(O.mafat_cross(**dict(CROSS, **shape))), *dict(CALL, **call).values())


@pytest.mark.parametrize("shape, call, status", [
    (dict(dtype=F8), {}, EUNSUPPORTED), (dict(frames=0), {}, EINVAL), (dict(rows=-1), {}, EINVAL),
    (dict(positions=-1), {}, EINVAL), (dict(q_heads=3), {}, EINVAL), (dict(kv_heads=0), {}, EINVAL),
    (dict(q_heads=0), {}, EINVAL), (dict(head_dim=0), {}, EINVAL),
    (dict(head_dim=257, q_head=257, k_head=257, v_head=257, y_head=257, q_row=1028, y_row=1028, k_pos=514, v_pos=514,
          k_frame=20560, v_frame=20560), {}, EUNSUPPORTED),
    (dict(scale=float("inf")), {}, EINVAL), (dict(scale=float("nan")), {}, EINVAL),
    (dict(q_head=63), {}, EINVAL), (dict(k_head=0), {}, EINVAL), (dict(v_head=-64), {}, EINVAL), (dict(y_head=1), {}, EINVAL),
    (dict(q_row=10), {}, EINVAL), (dict(y_row=0), {}, EINVAL), (dict(k_pos=0), {}, EINVAL), (dict(v_frame=0), {}, EINVAL),
    (dict(mask_row=39), {}, EINVAL), (dict(mask_row=-1), {}, EINVAL),
    (dict(rows=1 << 30), {}, EUNSUPPORTED), (dict(positions=1 << 31), {}, EUNSUPPORTED),
    (dict(k_pos=1 << 30), {}, EUNSUPPORTED), (dict(q_row=1 << 30), {}, EUNSUPPORTED), (dict(k_frame=1 << 58), {}, EUNSUPPORTED),
    (dict(kv_heads=65536, q_heads=65536), {}, EUNSUPPORTED),
    (dict(rows=5), dict(q_offsets=None), EINVAL),
    ({}, dict(q=None), EINVAL), ({}, dict(k=None), EINVAL), ({}, dict(v=None), EINVAL), ({}, dict(y=None), EINVAL),
    ({}, dict(q=A + 1), EINVAL), (dict(dtype=F32), dict(k=B + 2), EINVAL), ({}, dict(q_offsets=C + 2), EINVAL),
    ({}, dict(k_lengths=C + 4097), EINVAL), ({}, dict(lse=D + (1 << 30) + 1), EINVAL),
    ({}, dict(y=A), EINVAL), ({}, dict(y=B + 2 * 40 * 256 * 2 - 2), EINVAL), ({}, dict(lse=D), EINVAL), ({}, dict(lse=C), EINVAL),
    (dict(positions=40000, k_frame=40000 * 256, v_frame=40000 * 256, mask_row=40000), dict(ws_bytes=0), M.MAFAT_EWORKSPACE),
    (dict(positions=40000, k_frame=40000 * 256, v_frame=40000 * 256, mask_row=40000), dict(workspace=None), EINVAL),
    (dict(positions=40000, k_frame=40000 * 256, v_frame=40000 * 256, mask_row=40000), dict(workspace=E + 16), EINVAL),
    (dict(positions=40000, k_frame=40000 * 256, v_frame=40000 * 256, mask_row=40000), dict(workspace=D), EINVAL),
])
def test_cross_refusals(shape, call, status):
    rc = _cross(shape, call)
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_cross_without_a_shape_or_rows():
    import ctypes
    assert O.lib().mafat_cross_attention(None, *CALL.values()) == EINVAL
    n = ctypes.c_size_t()
    assert O.lib().mafat_cross_workspace(None, ctypes.byref(n)) == EINVAL
    assert O.lib().mafat_cross_workspace(ctypes.byref(O.mafat_cross(**CROSS)), None) == EINVAL
    assert _cross(dict(rows=0), dict(q=None, y=None, workspace=None, ws_bytes=0)) == 0
