"""CPU tests of the C entries of the operators among a request's tokens (include/mafat_reader.h): each refusal comes back as
its status before any HIP call (pointers below are never followed)."""
import ctypes

import pytest

from paper_2107_06960_amd import mafat as M
from paper_2107_06960_amd import operators as O

EINVAL, EUNSUPPORTED = M.MAFAT_EINVAL, M.MAFAT_EUNSUPPORTED
F32, BF16, F8 = M.MAFAT_F32, M.MAFAT_BF16, O.MAFAT_F8
A, B, C, D, E, F, G, H = (k << 32 for k in range(1, 9))  # device addresses far apart
NAN, INF = float("nan"), float("inf")

TURNS = dict(dtype=BF16, axes=1, rows=4, q_heads=4, k_heads=2, head_dim=64, pairs=32, interleaved=0, magnitude=1.0, q_row=256,
             q_head=64, k_row=128, k_head=64, qy_row=256, qy_head=64, ky_row=128, ky_head=64)
ROTARY = dict(positions=A, turns=B, q=C, k=D, qy=E, ky=F, stream=None)


def _rotary(shape, call):
    return O.lib().mafat_rotary(ctypes.byref(O.mafat_turns(**dict(TURNS, **shape))), *dict(ROTARY, **call).values())


@pytest.mark.parametrize("shape, call, status", [
    (dict(dtype=F8), {}, EUNSUPPORTED), (dict(rows=-1), {}, EINVAL), (dict(q_heads=0), {}, EINVAL), (dict(k_heads=-1), {}, EINVAL),
    (dict(axes=0), {}, EINVAL), (dict(axes=5), {}, EINVAL), (dict(head_dim=0), {}, EINVAL), (dict(pairs=33), {}, EINVAL),
    (dict(pairs=-1), {}, EINVAL), (dict(pairs=1 << 30), {}, EINVAL), (dict(magnitude=NAN), {}, EINVAL), (dict(magnitude=INF), {}, EINVAL),
    (dict(head_dim=1025, q_row=4100, q_head=1025, k_row=2050, k_head=1025, qy_row=4100, qy_head=1025, ky_row=2050, ky_head=1025),
     {}, EUNSUPPORTED),
    (dict(rows=1 << 31), {}, EUNSUPPORTED), (dict(q_heads=65536), {}, EUNSUPPORTED), (dict(k_heads=65536), {}, EUNSUPPORTED),
    (dict(q_row=63), {}, EINVAL), (dict(q_head=0), {}, EINVAL), (dict(k_row=-128), {}, EINVAL), (dict(ky_head=1), {}, EINVAL),
    (dict(q_row=1 << 31), {}, EUNSUPPORTED), (dict(ky_row=1 << 31), {}, EUNSUPPORTED),
    ({}, dict(positions=None), EINVAL), ({}, dict(turns=None), EINVAL), ({}, dict(q=None), EINVAL), ({}, dict(qy=None), EINVAL),
    ({}, dict(k=None), EINVAL), ({}, dict(ky=None), EINVAL), (dict(k_heads=0), {}, EINVAL), (dict(k_heads=0), dict(k=None), EINVAL),
    ({}, dict(positions=A + 2), EINVAL), ({}, dict(turns=B + 4), EINVAL), ({}, dict(q=C + 1), EINVAL), (dict(dtype=F32), dict(ky=F + 2), EINVAL),
    # overlaps: shifted on its own input, on the other input, on each other, on the positions and the table
    ({}, dict(qy=C + 2), EINVAL), ({}, dict(qy=D), EINVAL), ({}, dict(ky=C), EINVAL), ({}, dict(ky=E + 1536), EINVAL), ({}, dict(qy=A), EINVAL),
    ({}, dict(ky=B), EINVAL), (dict(qy_row=512), dict(qy=C), EINVAL),
])
def test_rotary_refusals(shape, call, status):
    rc = _rotary(shape, call)
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_rotary_without_rows():
    assert O.lib().mafat_rotary(None, *ROTARY.values()) == EINVAL
    assert _rotary(dict(rows=0), dict(positions=None, q=None, k=None, qy=None, ky=None)) == 0


BLOCK = dict(dtype=BF16, out_dtype=F8, rows=4, cols=64, after=1, groups=4, gate_act=1, before=1, eps=1e-6, x_stride=64,
             gate_stride=64, residual_stride=64, sum_stride=64, y_stride=64)
NORM = dict(x=A, after_gain=B, gate=C, scale=D, residual=E, sum=F, before_gain=G, y=H, y_scale=H + (1 << 31), stream=None)


def _block(shape, call):
    return O.lib().mafat_block_norm(ctypes.byref(O.mafat_block(**dict(BLOCK, **shape))), *dict(NORM, **call).values())


@pytest.mark.parametrize("shape, call, status", [
    (dict(dtype=F8), {}, EUNSUPPORTED), (dict(out_dtype=3), {}, EUNSUPPORTED), (dict(rows=-1), {}, EINVAL), (dict(cols=0), {}, EINVAL),
    (dict(rows=1 << 31), {}, EUNSUPPORTED), (dict(cols=1 << 31), {}, EUNSUPPORTED), (dict(groups=0), {}, EINVAL),
    (dict(groups=3), {}, EINVAL), (dict(groups=8192, cols=8192), {}, EUNSUPPORTED), (dict(eps=-1e-6), {}, EINVAL),
    (dict(eps=NAN), {}, EINVAL), (dict(eps=INF), {}, EINVAL), ({}, dict(residual=None), EINVAL), ({}, dict(sum=None), EINVAL),
    (dict(after=0), {}, EINVAL), (dict(before=0), {}, EINVAL), ({}, dict(y_scale=None), EINVAL), (dict(out_dtype=F32), {}, EINVAL),
    (dict(x_stride=63), {}, EINVAL), (dict(gate_stride=0), {}, EINVAL), (dict(residual_stride=1), {}, EINVAL),
    (dict(sum_stride=-64), {}, EINVAL), (dict(y_stride=63), {}, EINVAL), (dict(x_stride=1 << 31), {}, EUNSUPPORTED),
    (dict(gate_stride=1 << 31), {}, EUNSUPPORTED), ({}, dict(x=None), EINVAL), ({}, dict(y=None), EINVAL), ({}, dict(x=A + 1), EINVAL),
    ({}, dict(gate=C + 1), EINVAL), ({}, dict(scale=D + 2), EINVAL), ({}, dict(before_gain=G + 1), EINVAL),
    ({}, dict(y_scale=H + (1 << 31) + 2), EINVAL),
    # overlaps: also a sum on the residual, which is read again
    ({}, dict(y=A), EINVAL), ({}, dict(y=C), EINVAL), ({}, dict(sum=E), EINVAL), ({}, dict(sum=A + 2), EINVAL), ({}, dict(y=F), EINVAL),
    ({}, dict(y_scale=H), EINVAL), ({}, dict(y=B), EINVAL), ({}, dict(sum=D), EINVAL),
])
def test_block_norm_refusals(shape, call, status):
    rc = _block(shape, call)
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_block_norm_without_rows():
    assert O.lib().mafat_block_norm(None, *NORM.values()) == EINVAL
    assert _block(dict(rows=0), dict(x=None, y=None)) == 0


DECAY = dict(dtype=BF16, requests=2, rows=6, slots=5, q_heads=4, kv_heads=2, key_dim=64, value_dim=32, scale=0.125, decay_by_row=1,
             q_row=256, q_head=64, k_row=128, k_head=64, v_row=64, v_head=32, y_row=128, y_head=32, decay_row=2, state_slot=4096)
LONG = dict(rows=40000, q_heads=2)
CALL = dict(q=A, k=B, v=C, log_decay=D, offsets=D + (1 << 30), states=E, slots=D + (1 << 31), y=F, workspace=G, ws_bytes=1 << 40,
            stream=None)


def _decay(shape, call):
    return O.lib().mafat_decay_attention(ctypes.byref(O.mafat_decay(**dict(DECAY, **shape))), *dict(CALL, **call).values())


@pytest.mark.parametrize("shape, call, status", [
    (dict(dtype=F8), {}, EUNSUPPORTED), (dict(requests=0), {}, EINVAL), (dict(rows=-1), {}, EINVAL), (dict(slots=-1), {}, EINVAL),
    (dict(q_heads=3), {}, EINVAL), (dict(kv_heads=0), {}, EINVAL), (dict(q_heads=0), {}, EINVAL), (dict(key_dim=0), {}, EINVAL),
    (dict(value_dim=0), {}, EINVAL), (dict(key_dim=257), {}, EUNSUPPORTED), (dict(value_dim=257), {}, EUNSUPPORTED),
    (dict(scale=NAN), {}, EINVAL), (dict(scale=INF), {}, EINVAL), (dict(q_row=63), {}, EINVAL), (dict(k_head=0), {}, EINVAL),
    (dict(v_row=31), {}, EINVAL), (dict(y_head=-32), {}, EINVAL), (dict(decay_row=1), {}, EINVAL), (dict(state_slot=4095), {}, EINVAL),
    (dict(rows=1 << 30), {}, EUNSUPPORTED), (dict(requests=1 << 30), {}, EUNSUPPORTED), (dict(slots=1 << 31), {}, EUNSUPPORTED),
    (dict(kv_heads=65536, q_heads=65536, decay_row=65536, state_slot=65536 * 2048), {}, EUNSUPPORTED),
    (dict(q_row=1 << 30), {}, EUNSUPPORTED), (dict(decay_row=1 << 31), {}, EUNSUPPORTED), (dict(state_slot=1 << 58), {}, EUNSUPPORTED),
    (dict(rows=5), dict(offsets=None), EINVAL), ({}, dict(q=None), EINVAL), ({}, dict(k=None), EINVAL), ({}, dict(v=None), EINVAL),
    ({}, dict(log_decay=None), EINVAL), ({}, dict(y=None), EINVAL), ({}, dict(states=None), EINVAL), ({}, dict(q=A + 1), EINVAL),
    (dict(dtype=F32), dict(v=C + 2), EINVAL), ({}, dict(log_decay=D + 2), EINVAL), ({}, dict(states=E + 2), EINVAL),
    ({}, dict(slots=D + (1 << 31) + 1), EINVAL), ({}, dict(y=A), EINVAL), ({}, dict(y=C), EINVAL), ({}, dict(y=E), EINVAL),
    ({}, dict(states=B), EINVAL), ({}, dict(states=D), EINVAL), ({}, dict(y=D + (1 << 30)), EINVAL),
    (LONG, dict(ws_bytes=0), M.MAFAT_EWORKSPACE), (LONG, dict(workspace=None), EINVAL), (LONG, dict(workspace=G + 16), EINVAL),
    (LONG, dict(workspace=A), EINVAL), (LONG, dict(workspace=E), EINVAL), (LONG, dict(workspace=F), EINVAL),
])
def test_decay_refusals(shape, call, status):
    rc = _decay(shape, call)
    assert rc == status, O.lib().mafat_last_error()
    assert O.lib().mafat_last_error()


def test_decay_without_a_shape_or_rows():
    assert O.lib().mafat_decay_attention(None, *CALL.values()) == EINVAL
    n = ctypes.c_size_t()
    assert O.lib().mafat_decay_workspace(None, ctypes.byref(n)) == EINVAL
    assert O.lib().mafat_decay_workspace(ctypes.byref(O.mafat_decay(**DECAY)), None) == EINVAL
    assert _decay(dict(rows=0), dict(q=None, k=None, v=None, y=None, workspace=None, ws_bytes=0)) == 0
    assert O.mafat_decay_workspace(O.mafat_decay(**DECAY)) == 0
    assert O.mafat_decay_workspace(O.mafat_decay(**dict(DECAY, **LONG))) > 0


@pytest.mark.parametrize("stretch, trained", [(1.0, None), (4.0, None), (8.0, 4096)])
def test_rotary_turns(stretch, trained):
    """Against the definition, pair by pair."""
    import math
    pairs, base = 32, 10000.0
    got = O.rotary_turns(pairs, base, stretch, trained, device="cpu")
    for i in range(pairs):
        t = base ** (-i / pairs) / (2 * math.pi)
        keep = 0.0 if trained is None else min(max((t * trained - 1) / 31, 0), 1)
        assert abs(got[i].item() - (t * keep + t / stretch * (1 - keep))) <= 1e-15
