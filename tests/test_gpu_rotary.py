"""Rotary positions (mafat_rotary) against the formula in float64.

Bound, from the arithmetic: turns are brought below half a turn in float64; as a float32 the angle is off by 2^-24 of itself,
at most pi 2^-24, and sincospi by at most 4 units, 4 * 2^-23 of at most 1; the magnitude's product, the two products and the
sum round once each.  So a value is within (pi + 8 + 3) 2^-24 < 16 * 2^-24 of magnitude (|x1| + |x2|); bfloat16 adds half a
step, 2^-8 of the value."""
import math

import pytest

from gpu_util import require_gpu


def _formula(x, positions, turns, interleaved, magnitude):
    """(turned values, what their bounds are relative to)."""
    import torch
    x, pairs = x.double().cpu(), turns.shape[-1]
    positions = positions.double().cpu().reshape(x.shape[0], -1)
    t = positions @ turns.cpu().reshape(positions.shape[1], pairs)
    t = 2 * math.pi * (t - t.round())[:, None]
    one = torch.arange(pairs) * 2 if interleaved else torch.arange(pairs)
    two = one + (1 if interleaved else pairs)
    y, size = x.clone(), torch.zeros_like(x)
    y[..., one] = magnitude * (x[..., one] * t.cos() - x[..., two] * t.sin())
    y[..., two] = magnitude * (x[..., two] * t.cos() + x[..., one] * t.sin())
    size[..., one] = size[..., two] = abs(magnitude) * (x[..., one].abs() + x[..., two].abs())
    return y, size


def _check(got, x, positions, turns, interleaved, magnitude):
    want, size = _formula(x, positions, turns, interleaved, magnitude)
    rel = 2.0 ** -8 if x.element_size() == 2 else 0.0
    # (8 more for turns that the oracle's products form in another order: 2^-53 of up to 2^22 turns, 2 pi over)
    bad = (got.double().cpu() - want).abs() > 16 * 2.0 ** -24 * size + rel * want.abs() + 1e-38
    assert not bad.any(), bad.nonzero()[:4]
    d = 2 * turns.shape[-1]
    assert (got[..., d:].contiguous().view(-1) == x[..., d:].contiguous().view(-1)).all()


def _x(rows, heads, d, dtype, gen, pad=0, shift=0):
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    buf = torch.randn(shift + rows * (heads * d + pad), generator=gen).to(dt).cuda()
    return buf[shift:].view(rows, heads * d + pad)[:, :heads * d].view(rows, heads, d)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d, pairs", [(64, 32), (128, 64), (128, 32), (256, 128), (80, 24), (40, 11), (2, 1), (3, 1), (7, 0),
                                      (96, 48), (33, 9), (1024, 512), (1000, 3), (1, 0)])
def test_rotary_against_the_formula(d, pairs, interleaved, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(1000 * d + pairs)
    for rows, hq, hk, axes, magnitude, pad, shift in [(1, 1, 0, 1, 1.0, 0, 0), (67, 5, 2, 2, 1.3, 0, 0), (300, 3, 3, 4, 1.0, 3, 1),
                                                      (1000, 8, 1, 1, -0.5, 8, 0)]:
        q = _x(rows, hq, d, dtype, gen, pad, shift)
        k = _x(rows, hk, d, dtype, gen, pad + 1, shift) if hk else None
        positions = torch.randint(-(1 << 20), 1 << 20, (rows, axes), generator=gen, dtype=torch.int32).cuda()
        turns = O.rotary_turns(pairs, stretch=2.0, trained=4096) * (0.5 + torch.arange(axes, device="cuda")[:, None])
        qy, ky = O.rotary(q, positions, turns, k=k, interleaved=interleaved, magnitude=magnitude)
        _check(qy, q, positions, turns, interleaved, magnitude)
        assert (ky is None) == (k is None)
        if hk:
            _check(ky, k, positions, turns, interleaved, magnitude)
        q2, k2 = q.clone(), None if k is None else k.clone()
        got = O.rotary(q2, positions, turns, k=k2, interleaved=interleaved, magnitude=magnitude, in_place=True)
        assert got[0] is q2 and got[1] is k2 and torch.equal(q2, qy) and (k is None or torch.equal(k2, ky))


@pytest.mark.gpu
def test_farthest_positions_and_back():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(3)
    q = _x(6, 4, 64, "f32", gen)
    positions = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32, device="cuda")
    turns = O.rotary_turns(32)
    y, none = O.rotary(q, positions, turns)
    assert none is None and torch.equal(y[0], q[0])
    _check(y, q, positions, turns, False, 1.0)
    back, _ = O.rotary(y[:4], -positions[:4], turns)
    assert ((back - q[:4]).abs().max() <= 64 * 2.0 ** -24 * q.abs().max()).item()


@pytest.mark.gpu
def test_parts_of_one_projection_in_place():
    """q and k side by side in rows that also hold something else, which stays."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(4)
    rows, hq, hk, d = 130, 4, 2, 64
    x = torch.randn(rows, (hq + 2 * hk) * d, generator=gen).bfloat16().cuda()
    before = x.clone()
    q, k = x[:, :hq * d].view(rows, hq, d), x[:, hq * d:(hq + hk) * d].view(rows, hk, d)
    positions, turns = torch.arange(rows, dtype=torch.int32, device="cuda"), O.rotary_turns(20)
    want = O.rotary(q, positions, turns, k=k)
    O.rotary(q, positions, turns, k=k, in_place=True)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(x[:, (hq + hk) * d:], before[:, (hq + hk) * d:])
    # heads outside of rows: [heads, rows, d] seen as [rows, heads, d]
    t = before[:, :hq * d].view(rows, hq, d).transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(O.rotary(t, positions, turns)[0], want[0])


@pytest.mark.gpu
def test_no_rows_nan_and_large_values_stay_theirs():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(5)
    turns = O.rotary_turns(16)
    empty, _ = O.rotary(torch.empty(0, 2, 64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), turns)
    assert empty.shape == (0, 2, 64)
    q = _x(9, 2, 64, "f32", gen)
    positions = torch.arange(9, dtype=torch.int32, device="cuda")
    clean, _ = O.rotary(q, positions, turns)
    q[3, 1, 5], q[4, 0, 40], q[5, 0, 63] = float("nan"), float("inf"), float("-inf")
    y, _ = O.rotary(q, positions, turns)
    touched = torch.zeros_like(q, dtype=torch.bool)
    touched[3, 1, 5] = touched[3, 1, 21] = touched[4, 0, 40] = touched[5, 0, 63] = True  # (40 and 63 are behind the pairs)
    assert torch.isnan(y[3, 1, 5]) and torch.isnan(y[3, 1, 21]) and y[4, 0, 40] == float("inf") and y[5, 0, 63] == float("-inf")
    assert torch.equal(y[~touched], clean[~touched])


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(6)
    q, k = _x(4, 2, 64, "bf16", gen), _x(4, 1, 64, "bf16", gen)
    p, t = torch.arange(4, dtype=torch.int32, device="cuda"), O.rotary_turns(32)
    for args, kw in [((q.half(), p, t), {}), ((q.cpu(), p, t), {}), ((q[0], p, t), {}), ((q, p.long(), t), {}), ((q, p[:3], t), {}),
                     ((q, p.cpu(), t), {}), ((q, p, t.float()), {}), ((q, p, t.cpu()), {}), ((q, p, t[None].expand(2, 32)), {}),
                     ((q, p[:, None].expand(4, 2).contiguous(), t), {}), ((q.transpose(1, 2), p, t), {}), ((q, p, t), {"k": k.float()}),
                     ((q, p, t), {"k": k[:3]}), ((q, p, t), {"k": k[..., :32]}), ((q, p, t), {"k": k[:, :0]})]:
        with pytest.raises(ValueError):
            O.rotary(*args, **kw)
    for args, kw in [((q, p, O.rotary_turns(33)), {}), ((q, p, t), {"magnitude": float("nan")}),
                     ((q, p[:, None].expand(4, 5).contiguous(), t[None].expand(5, 32).contiguous()), {}),
                     ((q[:1].expand(4, 2, 64), p, t), {"in_place": True})]:
        with pytest.raises(M.MafatError):
            O.rotary(*args, **kw)
    with pytest.raises(ValueError, match="forward only"):
        O.rotary(q.float().requires_grad_(), p, t)


@pytest.mark.gpu
def test_runs_on_the_current_stream_and_replays():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gen = torch.Generator().manual_seed(7)
    q, k = _x(50, 4, 64, "bf16", gen), _x(50, 2, 64, "bf16", gen)
    p, t = torch.arange(50, dtype=torch.int32, device="cuda"), O.rotary_turns(32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        O.rotary(q, p, t, k=k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = O.rotary(q, p, t, k=k)
    for i in range(3):
        p.add_(1000 * i)
        q.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        want = O.rotary(q, p, t, k=k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
