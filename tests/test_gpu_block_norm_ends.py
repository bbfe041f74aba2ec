"""Norms around a block where float32 ends and where a step's rounding can be told: the largest 8-bit rows, gates that
nearly close, parts without a floor, and norms whose sums are exact.

Where every sum is exact the result is that of float32's own divisions and roots (correctly rounded, as numpy's are), bit by
bit, on every kernel and as add_rms_norm has it."""
import numpy as np
import pytest

from gpu_util import require_gpu
from test_gpu_block_norm import E, _check

# columns of every kernel: parts of a wave, waves, two pieces a thread, rows that are read again
WIDTHS = [8, 64, 100, 512, 1000, 2048, 4096, 8192, 16384, 40004]


def _signs(rows, cols, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 2, (rows, cols), generator=g).float() * 2 - 1


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


def _inverse_root(sq, n, eps):
    """1 / sqrt(sq / n + eps), each step rounded to float32."""
    return np.float32(1) / np.sqrt(np.float32(sq) / np.float32(n) + np.float32(eps))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", WIDTHS)
def test_norms_divide_and_take_roots(cols):
    """Rows of plus and minus one number (powers of two times 1, 3 or 5): their sums of squares are exact in any order."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    sizes = torch.tensor([1.0, 3.0, 5.0, 0.375, 96.0, 2.0 ** -20, 5 * 2.0 ** 30, 0.0])
    x = _signs(len(sizes), cols, cols) * sizes[:, None]
    x[:, ::3] = 0  # the mean is not the square
    sq = (x.double() ** 2).sum(1).numpy()
    assert (np.float32(sq) == sq).all()
    for eps in (1e-6, 0.3):
        want = x * torch.from_numpy(_inverse_root(sq, cols, eps))[:, None]
        for kw in (dict(after=True, before=False), dict(after=False, before=True)):
            got = O.block_norm(x.cuda(), eps=eps, out="f32", **kw)[1]
            assert torch.equal(got.cpu(), want), (kw, (got.cpu() - want).abs().max())
        assert torch.equal(O.add_rms_norm(x.cuda(), eps=eps, out="f32")[1].cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("cols, groups", [(64, 8), (4096, 32), (8192, 64), (16384, 128), (96, 4), (960, 5), (9600, 3), (16320, 20),
                                          (33, 3), (40, 40), (1000, 8), (40000, 10)])
def test_norms_of_parts_divide_and_take_roots(cols, groups):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _signs(6, cols, cols) * torch.tensor([1.0, 3.0, 5.0, 0.375, 2.0 ** -20, 5 * 2.0 ** 30])[:, None]
    x[:, ::5] = 0
    parts = x.view(6, groups, -1)
    sq = (parts.double() ** 2).sum(2).numpy()
    assert (np.float32(sq) == sq).all()
    for eps in (1e-6, 0.3):
        inv = torch.from_numpy(_inverse_root(sq, cols // groups, eps))
        got = O.block_norm(x.cuda(), groups=groups, eps=eps, before=False, out="f32")[1]
        assert torch.equal(got.cpu(), (parts * inv[..., None]).view(6, cols))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 40004])
@pytest.mark.parametrize("act", ["silu", "sigmoid"])
def test_gates_that_nearly_close(act, cols):
    """From where the exponential is near float32's end to where the gate is zero: values below 2^-126 are off by half of float32's
    least step, 2^-149, a factor of 2 for x and a second rounding; the others by 8 units."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gate = torch.linspace(-120, -60, cols).view(1, cols).cuda()
    x = torch.full_like(gate, 2.0)
    _, y, _ = O.block_norm(x, after=False, gate=gate, act=act, before=False, out="f32")
    g = gate.double()
    want = 2 * (g if act == "silu" else 1) / (1 + torch.exp(-g))
    assert ((y.double() - want).abs() <= 16 * E * want.abs() + 2 * 2.0 ** -149).all(), ((y.double() - want) / want).abs().max()
    far = torch.tensor([[-float("inf"), -1e30, float("nan"), float("inf"), 1e30, -111.0, -104.0, 3.0]], device="cuda")
    got = O.block_norm(torch.ones_like(far), after=False, gate=far, act=act, before=False, out="f32")[1]
    want = (far if act == "silu" else 1) / (1 + torch.exp(-far.double()))
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert ((got.double() == want) | ((got.double() - want).abs() <= 16 * E * want.abs() + 2.0 ** -149))[fine].all(), (got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols, groups", [(768, 12), (96, 4), (64, 8), (480, 15), (2560, 20), (5120, 40), (9600, 75), (960, 5), (9600, 3),
                                          (16320, 20), (33, 3), (1000, 8), (40000, 10), (100, 1), (1000, 1)])
def test_parts_without_a_floor(cols, groups, dtype):
    """eps = 0: rows and parts that are not zeros have their norm, whatever their team's threads past the row's end hold."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    g = torch.Generator().manual_seed(cols)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, gate, res = ((torch.randn(5, cols, generator=g) + 0.1).to(dt).cuda() for _ in range(3))
    for kw in (dict(before=True, out="f8"), dict(before=False, out="f8"), dict(before=True, out=dtype, residual=res, gate=gate)):
        args = dict(dict(x=x, after=True, after_gain=None, groups=groups, gate=None, act="silu", scale=None, residual=None, before=True,
                         before_gain=None, eps=0.0, out="f8"), **kw)
        result = O.block_norm(**args)
        assert torch.isfinite(result[1].float()).all()
        _check(args, result)
