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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, rows, cols, residual", [("f32", 2 ** 28 + 9, 1, True), ("bf16", 2 ** 26 + 5, 129, False),
                                                         ("bf16", 2 ** 24 + 3, 1025, False), ("bf16", 2 ** 22 + 3, 8200, False)])
def test_norm_of_rows_past_a_launch(dtype, rows, cols, residual):
    """Each number of threads per row with 2^32 threads and a few blocks more; all rows but a few are zeros."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.zeros(rows, cols, dtype=dt, device="cuda")
    at = torch.tensor([0, 1, rows // 2 - 1, rows // 2, rows - 12, rows - 2, rows - 1], device="cuda")
    torch.manual_seed(cols)
    x[at] = torch.randn(len(at), cols, device="cuda").to(dt)
    r = torch.ones(rows, cols, dtype=dt, device="cuda") if residual else None
    h, y, scale = O.add_rms_norm(x, None, r)
    small = O.add_rms_norm(x[at], None, r[at] if residual else None)
    assert torch.equal(y[at].view(torch.uint8), small[1].view(torch.uint8)) and torch.equal(scale[at], small[2])
    if residual:
        assert torch.equal(h[at], small[0]) and int((h == 1).sum()) == rows - len(at)
    rest = 1 / 448 if residual else 1.0  # the scale of a row of ones, of a row of zeros
    near = ((scale - rest).abs() < 1e-6).sum() - ((small[2] - rest).abs() < 1e-6).sum()
    assert int(near) == rows - len(at)


@pytest.mark.gpu
@pytest.mark.parametrize("rows, k, n, adapters", [(2 ** 24 + 5, 17, 3, 2), (2 ** 29 + 37, 16, 1, 1), (2 ** 31 - 1, 16, 1, 0)])
def test_linear_of_rows_past_a_launch(rows, k, n, adapters):
    """Each way of the adapters' inner products, and the tiles, with 2^32 threads and more; all rows but a few are zeros."""
    require_gpu()
    import torch
    import test_gpu_linear as L
    from paper_2107_06960_amd import operators as O
    at = torch.tensor([0, 1, 2 ** 22 - 257, 2 ** 22 - 256, rows // 2, rows - 40, rows - 2, rows - 1], device="cuda")
    sx, sxs, w, ws, bias, ad, of = L._make(len(at), k, n, adapters, 3, k)
    x = torch.zeros(rows, k, dtype=torch.uint8, device="cuda")
    x[at] = sx.contiguous().view(torch.uint8)
    xs = torch.ones(rows, device="cuda")
    xs[at] = sxs
    of_row = None
    if adapters:
        of_row = torch.full((rows,), adapters - 1, dtype=torch.int32, device="cuda")
        of_row[at] = of
    y = O.linear8(x.view(O.F8), xs, w, ws, bias, ad, of_row)
    L._check(y[at], (sx, sxs, w, ws, bias, ad, of))
    for j in range(n):  # zeros give the bias
        assert rows - len(at) <= int((y[:, j] == bias[j].bfloat16()).sum()) <= rows


@pytest.mark.gpu
@pytest.mark.parametrize("frames, each, d", [(2 ** 24 + 3, 1, 8), (2 ** 24 + 3, 1, 7), (2 ** 23 + 1, 65, 8)])
def test_cross_attention_of_frames_past_a_launch(frames, each, d):
    """The kernels for few rows, for any size and for many rows with 2^32 threads and a few blocks more.  Frames of one
    position: every row gets its frame's value as it is."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    torch.manual_seed(d)
    v = torch.randn(frames, 1, 1, d, device="cuda").bfloat16()
    q = torch.ones(frames * each, 1, d, dtype=torch.bfloat16, device="cuda")
    y, _ = O.cross_attention(q, v, v)
    assert torch.equal(y.view(frames, each, d), v.view(frames, 1, d).expand(frames, each, d))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, d, mask", [(3, 128, "keys"), (100, 128, "keys"), (3, 127, "keys"), (520, 128, "rows"),
                                           (520, 127, "rows")])
def test_frames_past_2_31_elements(rows, d, mask):
    """The kernels for few rows, many rows and any size; keys and values of 2.2e9 elements in rows of 512, and masks of 2.2e9
    bytes where a row has its own.  Read are some positions at the start, around 2^30 and 2^31 elements and at the end."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    s = 4_300_000
    assert s * 512 > 2 ** 31
    at = torch.cat([torch.arange(20), torch.arange(2 ** 21 - 20, 2 ** 21 + 20), torch.arange(2 ** 22 - 20, 2 ** 22 + 20),
                    torch.arange(s - 200, s)]).cuda()
    kv = torch.zeros(1, s, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
    torch.manual_seed(rows + d)
    kv[:, at] = torch.randn(1, len(at), 2, 2, 128, device="cuda").bfloat16()
    k, v = kv[:, :, 0, :, :d], kv[:, :, 1, :, :d]
    q = torch.randn(rows, 2, d, device="cuda").bfloat16()
    some = torch.rand(rows if mask == "rows" else 1, len(at), device="cuda") < 0.8
    m = torch.zeros(len(some), s, dtype=torch.bool, device="cuda")
    m[:, at] = some
    name = {"keys": "key_mask", "rows": "row_mask"}[mask]
    got, lse = O.cross_attention(q, k, v, lse=True, **{name: m})
    pick = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda").unique()
    small = {"q": q[pick], "k": k[:, at], "v": v[:, at], name: some[pick] if mask == "rows" else some}
    y, allowed, want_lse, lse_allowed = _formula(small)
    assert torch.all((got[pick].double().cpu() - y).abs() <= allowed)
    assert torch.all((lse[pick].double().cpu() - want_lse).abs() <= lse_allowed)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [2048, 2047])
def test_linear_past_2_31_elements(k):
    """x and y of more than 2^31 elements each, on the tiles and on the kernel for any size."""
    require_gpu()
    import torch
    import test_gpu_linear as L
    from paper_2107_06960_amd import operators as O
    rows, n = 1_100_000, 2000
    assert rows * k > 2 ** 31 and rows * n > 2 ** 31
    at = torch.cat([torch.arange(3), torch.arange(rows // 2, rows // 2 + 30), torch.arange(rows - 70, rows)]).cuda()
    sx, sxs, w, ws, bias, ad, of = L._make(len(at), k, n, 3, 20, k)
    x = torch.zeros(rows, k, dtype=torch.uint8, device="cuda")
    x[at] = sx.contiguous().view(torch.uint8)
    xs = torch.ones(rows, device="cuda")
    xs[at] = sxs
    of_row = torch.full((rows,), 1, dtype=torch.int32, device="cuda")
    of_row[at] = of
    y = O.linear8(x.view(O.F8), xs, w, ws, bias, ad, of_row)
    L._check(y[at], (sx, sxs, w, ws, bias, ad, of))
    rest = torch.arange(5, rows, 9973, device="cuda")
    rest = rest[~torch.isin(rest, at)]
    assert torch.equal(y[rest], bias.bfloat16().expand(len(rest), n))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, cols", [(530_000, 4096), (60_000, 36_000)])
def test_norm_past_2_31_elements(rows, cols):
    """Rows that stay in registers and rows that are read again."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    assert rows * cols > 2 ** 31
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    torch.manual_seed(cols)
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    r = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[at] = torch.randn(len(at), cols, device="cuda").bfloat16()
    h, y, scale = O.add_rms_norm(x, None, r)
    small = O.add_rms_norm(x[at], None, r[at])
    assert torch.equal(h[at], small[0]) and torch.equal(y[at].view(torch.uint8), small[1].view(torch.uint8))
    assert torch.equal(scale[at], small[2])
    rest = torch.arange(7, rows - 7, 997, device="cuda")
    rest = rest[~torch.isin(rest, at)]
    assert (h[rest] == 2).all() and (y[rest].float() == 448).all()
