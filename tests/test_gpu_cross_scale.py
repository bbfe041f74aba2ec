"""Scales of cross attention (mafat_cross_attention) at the ends of their range and between calls; bounds as in
test_gpu_cross.py."""
import pytest

from gpu_util import require_gpu
from test_gpu_cross import _make


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
