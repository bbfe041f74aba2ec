"""Where cross attention in bfloat16 may not lose bits, whichever kernel runs.  The log-sum-exp is a float32 sum of float32
exponentials, so within the bound of the scores and of float32 (test_gpu_cross.py) without the rounding of the exponentials
that the second product takes; with few rows that product does not take it either."""
import math

import pytest

from gpu_util import require_gpu
from test_gpu_cross import _formula, _make


@pytest.mark.gpu
@pytest.mark.parametrize("d, shift, pad", [(64, 0, 0), (33, 0, 0), (7, 1, 0), (64, 1, 0), (128, 3, 5), (250, 0, 0)])
@pytest.mark.parametrize("rows, s", [(2, 4), (3, 70), (2, 3000), (150, 5), (150, 400)])
def test_lse_in_float32(rows, s, d, shift, pad):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    for mask in ("none", "keys", "rows"):
        a = _make(1, rows, s, 2, 1, d, "bf16", rows + s + d, mask=mask, shift=shift, pad=pad)
        _, lse = O.cross_attention(**a, lse=True)
        _, _, want, allowed = _formula(a)
        none = want == -math.inf
        lse = lse.double().cpu()
        assert torch.equal(lse == -math.inf, none)
        diff = (lse - want).abs()[~none] - (allowed - 2.0 ** -8)[~none]
        assert diff.numel() == 0 or diff.max() <= 0, float(diff.max())


@pytest.mark.gpu
@pytest.mark.parametrize("d, shift, pad", [(64, 0, 0), (33, 0, 0), (7, 1, 0), (64, 1, 0), (128, 3, 5), (250, 0, 0)])
@pytest.mark.parametrize("rows, s", [(2, 4), (3, 70), (2, 3000)])
def test_few_rows_do_not_round_the_exponentials(rows, s, d, shift, pad):
    """They enter the second product as two bfloat16 parts, 2^-16 of them lost at most, on every kernel."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(1, rows, s, 2, 1, d, "bf16", rows + s + d, shift=shift, pad=pad)
    got, _ = O.cross_attention(**a)
    y, allowed, _, _ = _formula(a)
    size = _formula(dict(a, v=a["v"].abs()))[0]  # sum p |v|, of which the bound has 2^-8 twice
    assert torch.all((got.double().cpu() - y).abs() <= allowed - 2 * (2.0 ** -8 - 2.0 ** -16) * size)
