"""The kernels that only large calls reach: the projection's tiles of 128 and 256, and cross attention's blocks of eight
waves with heads up to 128.  Bounds as in test_gpu_linear.py and test_gpu_cross.py."""
import math

import pytest

import test_gpu_linear as L
from gpu_util import require_gpu
from test_gpu_cross import _make


def _side(rows, n):
    """The tile that the projection's rule takes: the largest of which there are 256."""
    return next((t for t in (256, 128) if -(-rows // t) * -(-n // t) >= 256), 64)


# ends inside of tiles, steps and 8 columns; one stage of k, two, and many
TILES = [(256, 4100, 1040, 4010), (256, 4096, 16, 4104), (256, 33000, 144, 300), (128, 2100, 1040, 2000), (128, 2048, 272, 2048),
         (128, 20000, 144, 250), (128, 300, 16, 11003)]


@pytest.mark.gpu
@pytest.mark.parametrize("side, rows, k, n", TILES)
def test_large_tiles(side, rows, k, n):
    require_gpu()
    from paper_2107_06960_amd import operators as O
    assert _side(rows, n) == side
    x, xs, w, ws, bias, _, _ = args = L._make(rows, k, n, 0, 0, rows + k)
    L._check(O.linear8(x, xs, w, ws, bias=bias), args)


@pytest.mark.gpu
@pytest.mark.parametrize("count, rank, grouped", [(1, 1, True), (16, 16, False), (5, 20, False), (3, 128, True)])
@pytest.mark.parametrize("side, rows, k, n", [t for t in TILES if t[1] < 10000])
def test_large_tiles_with_adapters(side, rows, k, n, count, rank, grouped):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, ad, of_row = L._make(rows, k, n, count, rank, rows + rank)
    if grouped:
        of_row = torch.sort(of_row).values
    L._check(O.linear8(x, xs, w, ws, bias, ad, of_row), (x, xs, w, ws, bias, ad, of_row))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, n", [(4100, 4010), (2100, 2000)])
def test_large_tiles_strided_with_nan_and_replayed(rows, n):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, xs, w, ws, bias, ad, _ = L._make(rows, 256, n, 4, 16, rows, pad=16)
    of_row = (torch.arange(rows) % 4).to(torch.int32).cuda()
    clean = O.linear8(x, xs, w, ws, bias, ad, of_row)
    L._check(clean, (x, xs, w, ws, bias, ad, of_row))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = O.linear8(x, xs, w, ws, bias, ad, of_row)
    for _ in range(3):
        got.zero_()
        assert torch.equal(O.linear8(x, xs, w, ws, bias, ad, of_row), clean)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, clean)
    xs[1] = float("nan")
    ws[7] = float("inf")
    ad[0][2, 3, 5] = float("nan")
    ad[1][3, :, 0] = float("inf")
    got = O.linear8(x, xs, w, ws, bias, ad, of_row)
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[1], touched[:, 7], touched[of_row >= 2] = True, True, True
    assert torch.equal(got[~touched], clean[~touched])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[of_row >= 2].float()).any()


def _formula(a):
    """(y, allowed error of y, lse, allowed error of lse) in float64, a frame and a head at a time."""
    import torch
    q, k, v = (a[n].double().cpu() for n in ("q", "k", "v"))
    bf16 = a["q"].dtype == torch.bfloat16
    rows, hq, d = q.shape
    frames, s, hkv, _ = k.shape
    off = a.get("q_offsets")
    off = [i * rows // frames for i in range(frames + 1)] if off is None else off.tolist()
    lens = [s] * frames if a.get("k_lengths") is None else a["k_lengths"].tolist()
    y, allowed = torch.zeros_like(q), torch.zeros_like(q)
    lse, lse_allowed = torch.full((rows, hq), -math.inf, dtype=torch.float64), torch.zeros(rows, hq, dtype=torch.float64)
    for f in range(frames):
        n, at = lens[f], slice(off[f], off[f + 1])
        ok = torch.ones(off[f + 1] - off[f], n, dtype=torch.bool)
        if a.get("key_mask") is not None:
            ok &= a["key_mask"][f, :n].cpu()
        if a.get("row_mask") is not None:
            ok &= a["row_mask"][at, :n].cpu()
        some = ok.any(1)
        if not some.any():
            continue
        for h in range(hq):
            kk, vv, qq = k[f, :n, h // (hq // hkv)], v[f, :n, h // (hq // hkv)], q[at, h]
            z = (qq @ kk.t()) / math.sqrt(d)
            size = (qq.abs() @ kk.abs().t()) / math.sqrt(d)
            ez = 2.0 ** -20 * (size * ok).amax(1) + 2.0 ** -22 * (z.abs() * ok).amax(1)
            z = z.masked_fill(~ok, -math.inf)
            p = torch.where(some[:, None], torch.softmax(z, 1), 0.0)
            y[at, h] = p @ vv
            rel = 2 * ez + 2.0 ** -20 + (2.0 ** -8 if bf16 else 0)
            allowed[at, h] = 2 * rel[:, None] * (p @ vv.abs()) + (2.0 ** -8 if bf16 else 2.0 ** -22) * y[at, h].abs()
            lse[at, h] = torch.logsumexp(z, 1)
            lse_allowed[at, h] = rel - (2.0 ** -8 if bf16 else 0) + 2.0 ** -21 * lse[at, h].abs()
    return y, allowed, lse, lse_allowed


# eight waves from 256 blocks of 256 pairs of a row and a head on
WAVES8 = [(64, 2112, 100, 8, 4), (4, 8196, 130, 8, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["none", "keys", "rows"])
@pytest.mark.parametrize("d", [32, 64, 80, 96, 128])
@pytest.mark.parametrize("frames, rows, s, hq, hkv", WAVES8)
def test_blocks_of_eight_waves(frames, rows, s, hq, hkv, d, mask, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    pairs = -(-rows // frames) * (hq // hkv)
    assert pairs > 64 and frames * hkv * -(-pairs // 256) >= 256
    for ragged in (True, False):
        a = _make(frames, rows, s, hq, hkv, d, dtype, rows + d, ragged=ragged, mask=mask)
        got, lse = O.cross_attention(**a, lse=True)
        y, allowed, want_lse, lse_allowed = _formula(a)
        diff = (got.double().cpu() - y).abs()
        assert torch.all(diff <= allowed), float((diff - allowed).max())
        none = want_lse == -math.inf
        lse = lse.double().cpu()
        assert torch.equal(lse == -math.inf, none)
        assert torch.all((lse - want_lse)[~none].abs() <= lse_allowed[~none])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["keys", "rows"])
def test_eight_waves_what_is_masked_may_hold_anything(mask, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    frames, rows, s, hq, hkv = WAVES8[0]
    a = _make(frames, rows, s, hq, hkv, 128, dtype, 3, ragged=True, mask=mask)
    if mask == "rows":
        a["row_mask"][:, 3::7] = False  # positions that no row may read
    want = O.cross_attention(**a, lse=True)
    out = torch.arange(s, device="cuda") >= a["k_lengths"][:, None]
    if mask == "keys":
        out |= ~a["key_mask"]
    else:
        out[:, 3::7] = True
    bad = (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min)
    for i, w in enumerate(bad):
        pick = out & (torch.arange(s, device="cuda") % 4 == i)
        a["k"][pick], a["v"][pick] = w, bad[(i + 1) % 4]
    got = O.cross_attention(**a, lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
