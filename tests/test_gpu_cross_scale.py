"""Scales of cross attention (mafat_cross_attention) at the ends of their range and between calls; bounds as in
test_gpu_cross.py."""
import math

import pytest

from gpu_util import require_gpu
from test_gpu_cross import _check, _make


@pytest.mark.gpu
def test_a_scale_held_in_a_tensor_is_read_at_every_call():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(1, 5, 70, 2, 1, 64, "f32", 1)
    for scale in (torch.tensor(0.5), torch.nn.Parameter(torch.tensor(0.5), requires_grad=False),
                  torch.tensor(0.5, dtype=torch.float64, device="cuda")):
        for value in (0.5, 2.0, -0.125):
            scale.fill_(value)
            got, want = O.cross_attention(**a, scale=scale, lse=True), O.cross_attention(**a, scale=value, lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** -125, 1.6e-38, 1.2e-38, -1.2e-38, 1e-42, -2.0 ** -149])
@pytest.mark.parametrize("rows, s", [(2, 150), (2, 3000), (200, 150), (200, 3000)])
def test_scales_near_zero(rows, s, scale, dtype):
    """The mean of the values that may be read, whatever the number of rows and splits."""
    require_gpu()
    _check(_make(2, rows, s, 4, 2, 64, dtype, 7, ragged=True, mask="keys"), scale=scale)
    _check(_make(1, rows, s, 4, 2, 33, dtype, 7), scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 33])
@pytest.mark.parametrize("rows, s", [(6, 150), (6, 3000), (200, 150), (200, 3000)])
def test_scores_past_float32(rows, s, d, dtype):
    """Products within float32 that the scale takes past it: NaN above, and below as if not valid; the other rows as ever."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(1, rows, s, 2, 1, d, dtype, 5)
    a["k"].abs_().add_(0.1)
    small = a["q"].clone() * 1e-20
    want, want_lse = O.cross_attention(small, a["k"], a["v"], scale=1e20, lse=True)
    q = small.clone()
    q[1], q[3] = 1e20, -1e20
    y, lse = O.cross_attention(q, a["k"], a["v"], scale=1e20, lse=True)
    assert torch.isnan(y[1]).all() and torch.isnan(lse[1]).all()
    assert not y[3].any() and (lse[3] == -math.inf).all()
    others = [i for i in range(rows) if i not in (1, 3)]
    assert torch.isfinite(want).all() and torch.isfinite(want_lse).all()
    # rows of a wave rescale their sums together, so the last bits may differ
    assert (y[others].float() - want[others].float()).abs().max() <= 2.0 ** -7
    assert (lse[others] - want_lse[others]).abs().max() <= 2.0 ** -18 * want_lse.abs().max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 33])
@pytest.mark.parametrize("rows", [6, 200])
def test_a_scale_of_zero_keeps_nan(rows, d, dtype):
    """Zero times NaN or infinity; the other rows get the mean of the values."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(1, rows, 150, 2, 1, d, dtype, 5)
    want, want_lse = O.cross_attention(**a, scale=0.0, lse=True)
    a["q"][1, 0, 5], a["q"][3, 1, 30] = float("nan"), float("-inf")
    y, lse = O.cross_attention(**a, scale=0.0, lse=True)
    bad = torch.zeros(rows, 2, dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[3, 1] = True
    assert torch.isnan(y[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(y[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
