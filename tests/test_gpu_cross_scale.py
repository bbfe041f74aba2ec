"""Scales of cross attention (mafat_cross_attention) at the ends of their range and between calls; bounds as in
test_gpu_cross.py."""
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
