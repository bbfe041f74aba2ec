"""Rotary positions in place where queries, keys and values lie head by head in a projection's rows."""
import pytest

from gpu_util import require_gpu
from test_gpu_rotary import _check


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rows, heads, parts", "heads, rows, parts", "rows, parts, heads", "heads, parts, rows", "parts, rows, heads"])
@pytest.mark.parametrize("rows", [1, 70])
def test_in_place_in_any_order(order, rows, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    sizes = {"rows": rows, "heads": 5, "parts": 3}
    order = order.split(", ")
    gen = torch.Generator().manual_seed(rows)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.randn(*(sizes[n] for n in order), 64, generator=gen).to(dt).cuda()
    q, k, v = x.permute(*(order.index(n) for n in ("parts", "rows", "heads")), 3)
    before = [t.clone() for t in (q, k, v)]
    positions, turns = torch.arange(rows, dtype=torch.int32, device="cuda") * 7, O.rotary_turns(24)
    want = O.rotary(before[0], positions, turns, k=before[1])
    got = O.rotary(q, positions, turns, k=k, in_place=True)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, before[2])
    _check(q, before[0], positions, turns, False, 1.0)
    # fewer keys than queries, as far as they lie apart
    x.copy_(torch.randn(x.shape, generator=gen).to(dt))
    few, before = k[:, 1:3], [q.clone(), k[:, 1:3].clone()]
    want = O.rotary(before[0], positions, turns, k=before[1])
    O.rotary(q, positions, turns, k=few, in_place=True)
    assert torch.equal(q, want[0]) and torch.equal(few, want[1])
