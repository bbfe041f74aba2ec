"""Norms around a block where float32 ends and where a step's rounding can be told: the largest 8-bit rows.

Where every sum is exact the result is that of float32's own divisions (correctly rounded, as numpy's are), bit by bit, on
every kernel."""
import numpy as np
import pytest

from gpu_util import require_gpu

# columns of every kernel: parts of a wave, waves, two pieces a thread, rows that are read again
WIDTHS = [8, 64, 100, 512, 1000, 2048, 4096, 8192, 16384, 40004]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_rows_in_8_bits_at_the_ends_of_float32(cols, dtype):
    """y_scale is the row's largest magnitude over 448, and y what 448 over it brings into 8 bits: for largest magnitudes up to
    float32's last, and down to where the row counts as zeros."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    tops = [3e38, 1.9e38, 1.3e38, 8.6e37, 8.4e37, 1e37, 1e30, 1e10, 7.3, 1.0, 3e-7, 1e-20, 2.5e-30]
    g = torch.Generator().manual_seed(cols)
    x = torch.rand(len(tops), cols, generator=g) * 2 - 1
    x[:, cols // 2] = 1
    x = (x * torch.tensor(tops)[:, None]).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    _, y, scale = O.block_norm(x.cuda(), after=False, before=False)
    most = x.float().abs().amax(1).numpy()
    assert np.array_equal(scale.cpu().numpy(), most / np.float32(448))
    by = torch.from_numpy(np.float32(448) / most)
    assert torch.equal(y.cpu().float(), (x.float() * by[:, None]).to(torch.float8_e4m3fn).float())
