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
