"""The 8-bit projection with adapters (mafat_linear) against the formula in float64.

Bounds: the output's rounding to bfloat16 is 2^-8 of the value at most.  Before it, the 8-bit matrix instructions drop
bits of small products beside large ones: 1.5e-5 of the root of the sum of squared products on average (measured over
random operands), seven times that allowed for a single output.  The rest is float32: 2^-17 of the sums of magnitudes."""
import pytest

from gpu_util import require_gpu

MFMA_REL = 1e-4


def _make(rows, k, n, adapters, rank, seed, pad=0, shift=0):
    import torch
    from paper_2107_06960_amd import operators as O
    g = torch.Generator().manual_seed(seed)

    def f8(r, c):
        v = torch.randn(r, c, generator=g)
        s = v.abs().amax(1) / 448
        buf = torch.zeros(r * (c + pad) + shift).to(O.F8).cuda()
        t = buf[shift:].view(r, c + pad)[:, :c]
        t.copy_((v / s[:, None]).to(O.F8).cuda())
        return t, s.cuda()

    x, xs = f8(rows, k)
    w, ws = f8(n, k)
    ws = ws / k ** 0.5
    bias = torch.randn(n, generator=g).cuda()
    if not adapters:
        return x, xs, w, ws, bias, None, None
    a = (torch.randn(adapters, rank, k, generator=g) / k ** 0.5).bfloat16().cuda()
    b = (torch.randn(adapters, n, rank, generator=g) / rank ** 0.5).bfloat16().cuda()
    f = (0.5 + torch.rand(adapters, generator=g)).cuda()
    of_row = torch.randint(-1, adapters + 1, (rows,), generator=g, dtype=torch.int32).cuda()  # both ends are none
    return x, xs, w, ws, bias, (a, b, f), of_row


def _formula(x, xs, w, ws, bias, adapters, of_row):
    """(y, allowed error)"""
    import torch
    xd = x.float().double().cpu() * xs.double().cpu()[:, None]
    wd = w.float().double().cpu() * ws.double().cpu()[:, None]
    y = xd @ wd.t()
    err = MFMA_REL * (xd.square() @ wd.square().t()).sqrt()
    size = xd.abs() @ wd.abs().t()
    if bias is not None:
        y = y + bias.double().cpu()
        size = size + bias.abs().double().cpu()
    if adapters is not None:
        a, b, f = adapters
        for i in range(a.shape[0]):
            at = (of_row.cpu() == i).nonzero()[:, 0]
            fi = 1.0 if f is None else f[i].item()
            ad, bd = a[i].double().cpu(), b[i].double().cpu()
            y[at] += fi * (xd[at] @ ad.t()) @ bd.t()
            size[at] += abs(fi) * (xd[at].abs() @ ad.abs().t()) @ bd.abs().t()
    return y, 2.0 ** -8 * y.abs() + err + 2.0 ** -17 * size


def _check(got, args):
    import torch
    want, allowed = _formula(*args)
    diff = (got.float().double().cpu() - want).abs()
    assert torch.all(diff <= allowed), (diff / allowed).max()


SHAPES = [  # rows, in, out: each number of row tiles, ends inside of steps and tiles, single rows and columns
    (1, 16, 1), (1, 128, 16), (3, 1, 5), (4, 2048, 130), (16, 256, 48), (17, 129, 33), (31, 1000, 17), (32, 1024, 64),
    (33, 144, 100), (64, 4096, 96), (65, 1360, 257), (100, 96, 1001), (128, 512, 512), (129, 272, 255), (257, 1040, 300),
    (300, 4112, 70), (513, 640, 513), (1083, 1360, 129), (1100, 128, 1030)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows, k, n", SHAPES)
def test_linear_against_the_formula(rows, k, n):
    require_gpu()
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, _, _ = args = _make(rows, k, n, 0, 0, rows * 7 + k)
    _check(O.linear8(x, xs, w, ws, bias=bias), args)
    _check(O.linear8(x, xs, w, ws), (x, xs, w, ws, None, None, None))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, k, n", SHAPES)
def test_linear_with_adapters(rows, k, n):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    for count, rank, grouped in [(1, 1, False), (3, 8, False), (17, 16, True), (5, 20, True), (2, 64, False), (4, 128, True)]:
        x, xs, w, ws, bias, ad, of_row = _make(rows, k, n, count, rank, rows + k + rank)
        if grouped:
            of_row = torch.sort(of_row).values
        _check(O.linear8(x, xs, w, ws, bias, ad, of_row), (x, xs, w, ws, bias, ad, of_row))
    _check(O.linear8(x, xs, w, ws, None, (ad[0], ad[1], None), of_row), (x, xs, w, ws, None, (ad[0], ad[1], None), of_row))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, k, n, pad, shift", [(5, 100, 33, 3, 1), (40, 256, 64, 16, 0), (200, 256, 300, 7, 5),
                                                    (300, 512, 256, 16, 16), (300, 500, 256, 12, 0), (300, 512, 256, 0, 8)])
def test_strided_and_unaligned_operands(rows, k, n, pad, shift):
    require_gpu()
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, ad, of_row = args = _make(rows, k, n, 3, 12, rows, pad, shift)
    _check(O.linear8(x, xs, w, ws, bias, ad, of_row), args)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 40, 300])
def test_nan_stays_in_its_row_column_and_adapter(rows):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, ad, _ = _make(rows, 256, 200, 4, 16, rows)
    of_row = (torch.arange(rows) % 4).to(torch.int32).cuda()
    clean = O.linear8(x, xs, w, ws, bias, ad, of_row)
    xs[1] = float("nan")
    ws[7] = float("inf")
    ad[0][2, 3, 5] = float("nan")
    ad[1][3, :, 0] = float("inf")
    got = O.linear8(x, xs, w, ws, bias, ad, of_row)
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[1], touched[:, 7], touched[of_row >= 2] = True, True, True
    assert torch.equal(got[~touched], clean[~touched])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[of_row >= 2].float()).any()
    # an adapter that no row names may hold anything
    of_row[of_row >= 2] = -1
    again = O.linear8(x, xs, w, ws, bias, ad, of_row)
    assert torch.isfinite(again[of_row == 0][:, :7].float()).all() and torch.isfinite(again[of_row == -1][:, :7].float()).all()


@pytest.mark.gpu
def test_equal_calls_give_equal_bits_and_replay():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    for rows in (4, 70, 600):
        x, xs, w, ws, bias, ad, of_row = _make(rows, 1040, 520, 5, 16, rows)
        want = O.linear8(x, xs, w, ws, bias, ad, of_row)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = O.linear8(x, xs, w, ws, bias, ad, of_row)
        for _ in range(3):
            got.zero_()
            assert torch.equal(O.linear8(x, xs, w, ws, bias, ad, of_row), want)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, ad, of_row = _make(4, 64, 32, 2, 8, 0)
    for args in [(x.float(), xs, w, ws), (x, xs, w.float(), ws), (x, xs[:3], w, ws), (x, xs, w, ws[:5]), (x, xs, w[:, :32], ws),
                 (x.cpu(), xs, w, ws), (x, xs, w, ws, bias.double()), (x, xs, w, ws, None, ad), (x, xs, w, ws, None, None, of_row),
                 (x, xs, w, ws, None, ad, of_row.long()), (x, xs, w, ws, None, (ad[0].float(), ad[1], ad[2]), of_row),
                 (x, xs, w, ws, None, (ad[0], ad[1].transpose(1, 2), ad[2]), of_row), (x.t(), xs, w, ws)]:
        with pytest.raises(ValueError):
            O.linear8(*args)
    assert O.linear8(x[:0], xs[:0], w, ws).shape == (0, 32)
    assert torch.equal(O.linear8(x[:1], xs[:1], w, ws), O.linear8(x, xs, w, ws)[:1])
