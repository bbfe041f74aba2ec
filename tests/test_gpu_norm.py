"""Residual addition and RMS norm (mafat_add_rms_norm) against the formula in float64.

Bounds, from the arithmetic: the sum of squares of a row is a tree of float32 additions of depth below 64 and the norm a
handful of roundings after it, so a float32 value is within 64 * 2^-24 of the formula, relative; bfloat16 adds half of a
unit in 8 bits (2^-9 .. 2^-8 relative), e4m3 half of one in 4 bits (2^-4), or half of its smallest step (2^-10 scales).
The stored sum is the correctly rounded one, bit for bit."""
import numpy as np
import pytest

from gpu_util import require_gpu

F32_REL = 64 * 2.0 ** -24


def _tensors(rows, cols, dtype, seed, pad=0, shift=0):
    """Two matrices whose rows are `cols + pad` apart and start `shift` elements into their buffer, and a gain."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def one(by):
        buf = (by * torch.randn(rows * (cols + pad) + shift, generator=g)).to(dt).cuda()
        return buf[shift:].view(rows, cols + pad)[:, :cols]

    return one(1.0), one(2.0), (1 + 0.2 * torch.randn(cols, generator=g)).cuda()


def _formula(h, gain, eps):
    h = h.double().cpu().numpy()
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return y if gain is None else y * gain.double().cpu().numpy()


def _check(out, y, scale, want, f32_rel=F32_REL):
    got = y.float().double().cpu().numpy()
    if out == "f8":
        s = scale.double().cpu().numpy()[:, None]
        most = np.abs(want).max(1, keepdims=True)
        assert np.all(np.abs(s - most / 448) <= 2 * f32_rel * s)
        allowed = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s) * (1 + 1e-5) + 4 * f32_rel * np.abs(want)
        assert np.all(np.abs(got * s - want) <= allowed)
        assert np.all(np.abs(got).max(1) == 448)
    else:
        rel = f32_rel + (2.0 ** -8 if out == "bf16" else 0)
        assert np.all(np.abs(got - want) <= rel * np.abs(want) + 1e-37)


# every number of pieces per thread and team size, the lengths around them, one column, and rows read again
COLS = [1, 3, 8, 63, 64, 65, 127, 128, 129, 255, 257, 511, 512, 520, 1000, 1001, 1024, 1031, 2047, 2048, 2056, 4096, 4097,
        8192, 8200, 16384, 16385, 32768, 32776, 40001]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_norm_against_the_formula(cols, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    rows = 5 if cols > 2048 else 19
    for seed, (out, with_res, with_gain) in enumerate([("f8", True, True), (dtype, False, True), ("f8", False, False),
                                                       ("f32", True, False), ("bf16", True, True)]):
        x, r, gain = _tensors(rows, cols, dtype, 100 * cols + seed)
        h, y, scale = O.add_rms_norm(x, gain if with_gain else None, r if with_res else None, eps=1e-5, out=out)
        if with_res:
            assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
        else:
            assert h is None
        _check(out, y, scale, _formula(h if with_res else x, gain if with_gain else None, 1e-5))
        assert (scale is None) == (out != "f8")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols, pad, shift", [(256, 8, 0), (250, 7, 1), (1001, 23, 3), (4096, 1, 5), (33000, 5, 1)])
def test_strided_and_unaligned_rows(cols, pad, shift, dtype):
    require_gpu()
    from paper_2107_06960_amd import operators as O
    x, r, gain = _tensors(7, cols, dtype, cols + pad, pad, shift)
    for out in ("f8", dtype):
        h, y, scale = O.add_rms_norm(x, gain, r, out=out)
        _check(out, y, scale, _formula(h, gain, 1e-6))


@pytest.mark.gpu
def test_many_rows_and_one():
    require_gpu()
    from paper_2107_06960_amd import operators as O
    for rows, cols in [(1, 1024), (1, 4096), (16411, 40), (3001, 256), (0, 64)]:
        x, r, gain = _tensors(rows, cols, "bf16", rows)
        h, y, scale = O.add_rms_norm(x, gain, r)
        assert y.shape == (rows, cols) and scale.shape == (rows,)
        if rows:
            _check("f8", y, scale, _formula(h, gain, 1e-6))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 1000, 4096, 36000])
def test_rows_of_zeros_nan_and_infinities_stay_theirs(cols):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, r, gain = _tensors(8, cols, "f32", cols)
    clean = O.add_rms_norm(x, gain, r)
    x[1], r[1] = 0, 0
    x[3, cols // 2] = float("nan")
    x[5, cols - 1] = float("inf")
    r[6, 0] = float("-inf")
    x[2], r[2] = 1e-36, 0  # far below eps: zero in 8 bits
    h, y, scale = O.add_rms_norm(x, gain, r)
    yf = y.float()
    assert torch.equal(yf[1], torch.zeros_like(yf[1])) and scale[1] == 1
    assert scale[2] == 1 and torch.equal(yf[2].abs(), torch.zeros_like(yf[2]))
    for row in (3, 5, 6):
        assert torch.isnan(scale[row]) and torch.isnan(yf[row]).any()
    for row in (0, 4, 7):  # the others do not change
        assert torch.equal(yf[row], clean[1].float()[row]) and scale[row] == clean[2][row]
    assert torch.isnan(O.add_rms_norm(x, gain, r, out="f32")[1][3]).all()


@pytest.mark.gpu
def test_sum_in_place_through_the_c_entry():
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    for cols in (256, 1001, 5000, 40000):
        for on in ("x", "residual"):
            x, r, gain = _tensors(6, cols, "bf16", cols)
            h, y, scale = O.add_rms_norm(x, gain, r)
            y2, s2 = torch.empty_like(y), torch.empty_like(scale)
            target = x if on == "x" else r
            O.mafat_add_rms_norm(6, cols, M.MAFAT_BF16, x.data_ptr(), cols, r.data_ptr(), cols, gain.data_ptr(), 1e-6,
                                 target.data_ptr(), cols, O.MAFAT_F8, y2.data_ptr(), cols, s2.data_ptr(),
                                 M._stream_handle(None))
            torch.cuda.synchronize()
            assert torch.equal(target, h) and torch.equal(y2.float(), y.float()) and torch.equal(s2, scale)


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    x, r, gain = _tensors(4, 64, "bf16", 1)
    for args, kw in [((x.half(), gain, r), {}), ((x.cpu(), gain, r), {}), ((x, gain, r[:3]), {}), ((x, gain, r.float()), {}),
                     ((x, gain.bfloat16(), r), {}), ((x, gain[:63], r), {}), ((x.t(), None, None), {}),
                     ((x[:1].expand(4, 64), gain, r), {}), ((x, gain, r), {"out": "f16"}), ((x[0], gain, None), {})]:
        with pytest.raises(ValueError):
            O.add_rms_norm(*args, **kw)
    with pytest.raises(M.MafatError):
        O.add_rms_norm(x, gain, r, eps=-1.0)


@pytest.mark.gpu
def test_runs_on_the_current_stream_and_replays():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, r, gain = _tensors(9, 777, "bf16", 3)
    want = O.add_rms_norm(x, gain, r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        O.add_rms_norm(x, gain, r)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = O.add_rms_norm(x, gain, r)
    for _ in range(3):
        for t in got:
            t.view(torch.uint8).zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1].float(), want[1].float()) and torch.equal(got[2], want[2])
