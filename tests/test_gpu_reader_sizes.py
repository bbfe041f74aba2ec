"""The reader's operators at the ends of the sizes that their C entries take."""
import pytest

from gpu_util import require_gpu
from test_gpu_cross import _formula


@pytest.fixture(autouse=True)
def _release():
    """Tens of GB a test: hand them back."""
    yield
    import torch
    if torch.cuda.is_available():
        torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 70])
def test_a_key_mask_up_to_the_last_position_there_can_be(rows):
    """2^31 - 1 positions: the mask is looked at 4096 positions ahead, past its end (keys and values are one tensor)."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    s, d = 2 ** 31 - 1, 8
    at = torch.cat([torch.arange(40), torch.arange(2 ** 30 - 20, 2 ** 30 + 20), torch.arange(s - 300, s)]).cuda()
    k = torch.zeros(1, s, 1, d, dtype=torch.bfloat16, device="cuda")
    torch.manual_seed(rows)
    k[:, at] = torch.randn(1, len(at), 1, d, device="cuda").bfloat16()
    q = torch.randn(rows, 1, d, device="cuda").bfloat16()
    mask = torch.zeros(1, s, dtype=torch.bool, device="cuda")
    mask[:, at] = True
    got, lse = O.cross_attention(q, k, k, key_mask=mask, lse=True)
    y, allowed, want_lse, lse_allowed = _formula({"q": q, "k": k[:, at], "v": k[:, at]})
    assert torch.all((got.double().cpu() - y).abs() <= allowed)
    assert torch.all((lse.double().cpu() - want_lse).abs() <= lse_allowed)
