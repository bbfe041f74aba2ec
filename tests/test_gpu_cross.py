"""Cross attention (mafat_cross_attention) against the formula in float64.

Bounds.  A score is a float32 sum of d products: within 2^-20 of the sum of their magnitudes (16 units in the last place);
so is, relative, its exponential, times two for the largest one it is measured against, and 2^-20 for the exponential
itself.  The output's error is at most that share of sum p |v| for the numerator and again for the denominator.  bfloat16
adds 2^-8 of sum p |v| / sum p for each of the two where the exponentials are rounded, and 2^-8 of the output for its own
rounding."""
import math

import pytest

from gpu_util import require_gpu


def _make(frames, rows, s, hq, hkv, d, dtype, seed, ragged=False, mask="none", shift=0, pad=0):
    """Keys and values are the halves of one buffer of [frames, s, 2, hkv, d + pad] values that starts `shift` in."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def buf(*shape):
        n = math.prod(shape)
        return torch.randn(n + shift, generator=g).to(dt).cuda()[shift:].view(shape)

    kv = buf(frames, s, 2, hkv, d + pad)[..., :d]
    a = {"q": (2 * buf(rows, hq, d + pad))[..., :d], "k": kv[:, :, 0], "v": kv[:, :, 1]}
    if ragged:
        cut = torch.randint(0, rows + 1, (frames - 1,), generator=g, dtype=torch.int32)
        a["q_offsets"] = torch.sort(torch.cat([torch.tensor([0, rows], dtype=torch.int32), cut])).values.int().cuda()
        lens = torch.randint(0, s + 1, (frames,), generator=g, dtype=torch.int32)
        lens[0] = s
        a["k_lengths"] = lens.cuda()
    if mask == "keys":
        a["key_mask"] = (torch.rand(frames, s, generator=g) < 0.7).cuda()
    elif mask == "rows":
        m = torch.rand(rows, s, generator=g) < 0.3
        m[::3] = False  # rows that read nothing
        a["row_mask"] = m.cuda()
    return a


def _formula(a, scale=None):
    """(y, allowed error of y, lse, allowed error of lse) in float64."""
    import torch
    q, k, v = (a[n].double().cpu() for n in ("q", "k", "v"))
    bf16 = a["q"].dtype == torch.bfloat16
    rows, hq, d = q.shape
    frames, s, hkv, _ = k.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    off = a.get("q_offsets")
    off = [i * rows // frames for i in range(frames + 1)] if off is None else off.tolist()
    lens = [s] * frames if a.get("k_lengths") is None else a["k_lengths"].tolist()
    y, allowed = torch.zeros(rows, hq, d, dtype=torch.float64), torch.zeros(rows, hq, d, dtype=torch.float64)
    lse, lse_allowed = torch.full((rows, hq), -math.inf, dtype=torch.float64), torch.zeros(rows, hq, dtype=torch.float64)
    for f in range(frames):
        n = min(max(lens[f], 0), s)
        for i in range(off[f], off[f + 1]):
            ok = torch.ones(n, dtype=torch.bool)
            if a.get("key_mask") is not None:
                ok &= a["key_mask"][f, :n].cpu()
            if a.get("row_mask") is not None:
                ok &= a["row_mask"][i, :n].cpu()
            at = ok.nonzero()[:, 0]
            if not len(at):
                continue
            for h in range(hq):
                kk, vv, qq = k[f, at, h // (hq // hkv)], v[f, at, h // (hq // hkv)], q[i, h]
                z = scale * (kk @ qq)
                ez = 2.0 ** -20 * abs(scale) * (kk.abs() @ qq.abs()).max() + 2.0 ** -22 * z.abs().max()
                p = torch.softmax(z, 0)
                y[i, h], lse[i, h] = p @ vv, torch.logsumexp(z, 0)
                rel = 2 * ez + 2.0 ** -20 + (2.0 ** -8 if bf16 else 0)
                allowed[i, h] = 2 * rel * (p @ vv.abs()) + (2.0 ** -8 if bf16 else 2.0 ** -22) * y[i, h].abs()
                lse_allowed[i, h] = rel + 2.0 ** -21 * lse[i, h].abs()
    return y, allowed, lse, lse_allowed


def _check(a, scale=None):
    import torch
    from paper_2107_06960_amd import operators as O
    got, lse = O.cross_attention(**a, scale=scale, lse=True)
    y, allowed, want_lse, lse_allowed = _formula(a, scale)
    diff = (got.double().cpu() - y).abs()
    assert torch.all(diff <= allowed), float((diff - allowed).max())
    none = want_lse == -math.inf
    lse = lse.double().cpu()
    assert torch.equal(lse == -math.inf, none)
    assert torch.all((lse - want_lse)[~none].abs() <= lse_allowed[~none])
    only, _ = O.cross_attention(**a, scale=scale)
    assert torch.equal(only, got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 7, 8, 20, 32, 40, 64, 80, 96, 128, 200, 256])
def test_head_sizes(d, dtype):
    require_gpu()
    _check(_make(2, 6, 77, 4, 2, d, dtype, d))
    _check(_make(2, 70, 130, 2, 1, d, dtype, d, ragged=True, mask="keys"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("s", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 3001])
def test_numbers_of_positions(s, dtype):
    require_gpu()
    _check(_make(1, 1, s, 4, 4, 64, dtype, s))
    _check(_make(2, 20, s, 4, 2, 64, dtype, s, ragged=True))
    _check(_make(2, 10, s, 8, 1, 64, dtype, s, mask="keys"))
    _check(_make(1, 9, s, 2, 1, 128, dtype, s, mask="rows"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, hq, hkv", [(1, 1, 1), (1, 8, 1), (1, 48, 1), (3, 5, 5), (31, 3, 1), (33, 2, 1), (64, 2, 2),
                                           (65, 6, 3), (127, 1, 1), (129, 2, 1), (300, 4, 2)])
def test_rows_and_heads(rows, hq, hkv, dtype):
    require_gpu()
    _check(_make(1, rows, 100, hq, hkv, 64, dtype, rows))
    _check(_make(3, rows, 70, hq, hkv, 128, dtype, rows, ragged=True, mask="rows"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("frames", [1, 2, 63, 64, 65, 130])
def test_many_frames_some_without_rows_or_positions(frames, dtype):
    require_gpu()
    a = _make(frames, 90, 40, 2, 1, 32, dtype, frames, ragged=True, mask="keys")
    if frames > 1:
        a["k_lengths"][1] = 0
    _check(a)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift, pad", [(1, 0), (0, 1), (3, 5), (0, 8), (8, 0)])
@pytest.mark.parametrize("d", [33, 64])
def test_strides_and_alignment(shift, pad, d, dtype):
    require_gpu()
    _check(_make(2, 40, 100, 4, 2, d, dtype, shift + pad, ragged=True, mask="rows", shift=shift, pad=pad))
    _check(_make(2, 2, 500, 4, 2, d, dtype, shift + pad, shift=shift, pad=pad))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_before_positions_and_shared_keys(dtype):
    """k and v as [frames, heads, positions, d] in memory; v the same tensor as k."""
    require_gpu()
    a = _make(2, 12, 90, 4, 2, 64, dtype, 5)
    a["k"] = a["k"].transpose(1, 2).contiguous().transpose(1, 2)
    a["v"] = a["k"]
    _check(a)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, s", [(4, 200), (150, 200), (4, 5000)])
def test_what_is_masked_may_hold_anything(rows, s, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    bad = (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min)
    for mask in ("keys", "rows"):
        a = _make(2, rows, s, 4, 2, 64, dtype, s, ragged=True, mask=mask)
        a["k_lengths"][1] = s // 2
        if mask == "rows":
            a["row_mask"][:, 3::7] = False  # positions that no row may read
        want = O.cross_attention(**a, lse=True)
        a["k"][1, s // 2:], a["v"][1, s // 2:] = bad[0], bad[1]
        out = ~a["key_mask"] if mask == "keys" else torch.zeros(2, s, dtype=torch.bool, device="cuda")
        if mask == "rows":
            out[:, 3::7] = True
        for i, w in enumerate(bad):
            pick = out & (torch.arange(s, device="cuda") % 4 == i)
            a["k"][pick], a["v"][pick] = w, bad[(i + 1) % 4]
        got = O.cross_attention(**a, lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 140])
def test_scores_far_apart_and_equal(rows, dtype):
    """Scores of thousands, all equal, rising and falling along the positions: no overflow, no rescaling lost."""
    require_gpu()
    for kind in ("rising", "falling", "equal", "one"):
        import torch
        a = _make(1, rows, 600, 2, 1, 64, dtype, 3)
        ramp = torch.arange(600, device="cuda").float()[None, :, None, None] * 0.05
        if kind == "equal":
            a["k"][:] = a["k"][:, :1]
        elif kind == "one":
            a["k"][0, 417] = 30 * a["q"][0, 0]
        else:
            a["q"].fill_(1.0)
            a["k"].copy_((ramp if kind == "rising" else 30 - ramp).expand_as(a["k"]))
        _check(a, scale=1.0 if kind in ("rising", "falling") else None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 2.0])
@pytest.mark.parametrize("rows", [2, 200])
def test_scales(rows, scale, dtype):
    require_gpu()
    _check(_make(2, rows, 150, 4, 2, 64, dtype, 7, ragged=True, mask="keys"), scale=scale)


@pytest.mark.gpu
def test_offsets_and_lengths_out_of_range_stay_inside():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(3, 20, 50, 2, 1, 64, "bf16", 1)
    a["q_offsets"] = torch.tensor([-5, 7, 7, 90], dtype=torch.int32, device="cuda")
    a["k_lengths"] = torch.tensor([-3, 10, 1000], dtype=torch.int32, device="cuda")
    got, lse = O.cross_attention(**a, lse=True)
    b = dict(a, q_offsets=torch.tensor([0, 7, 7, 20], dtype=torch.int32, device="cuda"),
             k_lengths=torch.tensor([0, 10, 50], dtype=torch.int32, device="cuda"))
    want, want_lse = O.cross_attention(**b, lse=True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    assert not got[:7].any() and (lse[:7] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("positions", [30, 4000])
def test_rows_of_no_frame_are_not_written(positions):
    require_gpu()
    import ctypes
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    a = _make(2, 10, positions, 2, 1, 64, "bf16", 2)
    off = torch.tensor([2, 4, 8], dtype=torch.int32, device="cuda")
    want, _ = O.cross_attention(**a, q_offsets=off)
    y = torch.full((10, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    k = a["k"]
    c = O.mafat_cross(M.MAFAT_BF16, 2, 10, positions, 2, 1, 64, 0.125, 128, 64, k.stride(0), k.stride(1), k.stride(1),
                      k.stride(0), k.stride(1), k.stride(1), 128, 64, 0, 0)
    n = O.mafat_cross_workspace(c)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    O.mafat_cross_attention(c, a["q"].data_ptr(), k.data_ptr(), a["v"].data_ptr(), off.data_ptr(), None, None, y.data_ptr(),
                            None, ws.data_ptr(), n, M._stream_handle(None))
    torch.cuda.synchronize()
    assert torch.equal(y[2:8], want[2:8]) and (y[:2] == 7).all() and (y[8:] == 7).all()


@pytest.mark.gpu
def test_a_frame_past_32_bit_offsets():
    """Keys and values of 2.2e9 bytes in one buffer, the last positions of the last frame against the formula."""
    require_gpu()
    import torch
    s, hkv, d = 2_200_000, 2, 128
    kv = torch.zeros(1, s, 2, hkv, d, dtype=torch.bfloat16, device="cuda")
    kv[:, -300:] = torch.randn(1, 300, 2, hkv, d, device="cuda").bfloat16()
    a = {"q": torch.randn(3, 4, d, device="cuda").bfloat16(), "k": kv[:, :, 0], "v": kv[:, :, 1]}
    a["key_mask"] = torch.zeros(1, s, dtype=torch.bool, device="cuda")
    a["key_mask"][:, -300:] = True
    small = {"q": a["q"], "k": a["k"][:, -300:], "v": a["v"][:, -300:]}
    from paper_2107_06960_amd import operators as O
    got, lse = O.cross_attention(**a, lse=True)
    y, allowed, want_lse, lse_allowed = _formula(small)
    assert torch.all((got.double().cpu() - y).abs() <= allowed)
    assert torch.all((lse.double().cpu() - want_lse).abs() <= lse_allowed)


@pytest.mark.gpu
def test_equal_calls_give_equal_bits_and_replay():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    for rows, s, mask in [(2, 5000, "keys"), (300, 400, "none"), (40, 300, "rows")]:
        a = _make(2, rows, s, 4, 2, 128, "bf16", rows, ragged=True, mask=mask)
        want = O.cross_attention(**a, lse=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = O.cross_attention(**a, lse=True)
        for _ in range(3):
            got[0].zero_(), got[1].zero_()
            again = O.cross_attention(**a, lse=True)
            graph.replay()
            torch.cuda.synchronize()
            for x in (got, again):
                assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])


@pytest.mark.gpu
def test_no_rows_and_no_positions():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(2, 4, 10, 2, 1, 64, "bf16", 0)
    y, lse = O.cross_attention(a["q"][:0], a["k"], a["v"], lse=True)
    assert y.shape == (0, 2, 64) and lse.shape == (0, 2)
    y, lse = O.cross_attention(a["q"], a["k"][:, :0], a["v"][:, :0], lse=True)
    assert not y.any() and (lse == -math.inf).all()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    a = _make(2, 4, 10, 4, 2, 64, "bf16", 0)
    q, k, v = a["q"], a["k"], a["v"]
    mask = torch.ones(2, 10, dtype=torch.bool, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    for args, kw in [((q.half(), k, v), {}), ((q, k.float(), v), {}), ((q, k[:, :5], v), {}), ((q[:, :3], k, v), {}),
                     ((q[..., :32], k, v), {}), ((q.cpu(), k, v), {}), ((q, k, v), dict(q_offsets=off.long())),
                     ((q, k, v), dict(q_offsets=off[:2])), ((q, k, v), dict(k_lengths=off)),
                     ((q, k, v), dict(key_mask=mask.int())), ((q, k, v), dict(key_mask=mask[:1])),
                     ((q, k, v), dict(row_mask=mask)), ((q, k, v), dict(key_mask=mask, row_mask=mask)),
                     ((q.transpose(1, 2).contiguous().transpose(1, 2), k, v), {})]:
        with pytest.raises(ValueError):
            O.cross_attention(*args, **kw)
    from paper_2107_06960_amd import mafat as M
    with pytest.raises(M.MafatError):
        O.cross_attention(q[:3], k, v)  # rows do not divide by the frames
    with pytest.raises(M.MafatError):
        O.cross_attention(q, k, v, scale=float("nan"))
