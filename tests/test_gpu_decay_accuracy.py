"""How near linear attention with decays in bfloat16 comes to its formula in float64, on the matrix cores' kernel at its main
sizes: a token's output does not depend on how many others its call has, and loses no more than its own rounding does.

Bounds, with e = 2^-24, n the tokens of a request.  Scores, states where rows read them and weighted values enter products as
two bfloat16 parts each; a part's rounding is off by at most half a step, 2^-8, so two parts leave 2^-16 of each of the three,
and the product of two second parts that is left out is 2^-16 as well: 4 * 2^-16 at most.  Sums in float32 add
(dk + n + 64) e of their magnitudes singly and, as independent roundings, 4 sqrt(dk + n + 64) e of their norm (see
test_gpu_decay.py).  What an output is off by beyond half a step of bfloat16 at its value stays below these, singly relative
to the sum of magnitudes, as a whole relative to the norm.  (Scores rounded once are off by up to 2^-8: 30 times as much.)

Kept states are sums of n terms, which enter as three parts: at most 3 n roundings in float32, independent ones sqrt(3 n) e of
the norm as a whole, and 8 e for the weights (exponential 2 e, its exponent 2 e, the weight's product e, two rescalings e
each, and the three parts' 2^-24).  That is 1.3e-6 at n = 64, where two parts alone would leave up to 2^-16 of a term."""
import pytest

from gpu_util import require_gpu
from test_gpu_decay import E, _inputs, _norm


def _reference(x, off, scale, slots):
    """(y, states after, the sums of y's and the states' magnitudes) in float64 on the GPU, token after token."""
    import torch
    q, k, v, g = (x[n].double() for n in ("q", "k", "v", "log_decay"))
    rows, hq, _ = q.shape
    hkv, dv = v.shape[1:]
    a = g.clamp(max=0).exp()
    states = x["states"].double()
    y = torch.zeros(rows, hq, dv, dtype=torch.float64, device="cuda")
    ya = torch.zeros_like(y)
    for r in range(len(off) - 1):
        s = states[slots[r]].clone()
        sa = s.abs()
        for t in range(off[r], off[r + 1]):
            at = (a[t] if a.dim() == 2 else a)[:, None, None]
            kv = k[t][:, :, None] * v[t][:, None, :]
            s, sa = at * s + kv, at * sa + kv.abs()
            qt = q[t].view(hkv, -1, q.shape[2], 1)
            y[t] = scale * (qt * s[:, None]).sum(2).view(hq, dv)
            ya[t] = scale * (qt.abs() * sa[:, None]).sum(2).view(hq, dv)
        states[slots[r]] = s
    return y, states, ya


def _half_step(t):
    import torch
    return torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -126))) - 8)


def _check_outputs(x, off, slots, scale):
    from paper_2107_06960_amd import operators as O
    import torch
    dk, n = x["q"].shape[2], max(b - a for a, b in zip(off, off[1:]))
    want, states, size = _reference(x, off, scale, slots)
    kept = x["states"].clone()
    i32 = dict(dtype=torch.int32, device="cuda")
    y = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=kept, slots=torch.tensor(slots, **i32),
                          offsets=torch.tensor(off, **i32), scale=scale)
    over = ((y.double() - want).abs() - _half_step(want)).clamp(min=0)
    assert (over <= ((dk + n + 64) * E + 4 * 2.0 ** -16) * size).all(), (over / size).max()
    assert _norm(over) <= (4 * (dk + n + 64) ** 0.5 * E + 4 * 2.0 ** -16) * _norm(want), _norm(over) / _norm(want)
    err = _norm(kept.double() - states) / _norm(states)
    assert err <= 4 * (dk + n + 64) ** 0.5 * E + 2.0 ** -24, err


# rows, heads, sizes of a head: below and above 65536 rows times heads, one and several query heads a state
CALLS = [(300, 2, 2, 128, 128), (4100, 16, 16, 128, 128), (4100, 32, 16, 128, 128), (2200, 32, 32, 128, 64), (4100, 16, 16, 64, 64),
         (2100, 64, 32, 64, 128), (2200, 32, 32, 256, 256), (300, 4, 2, 256, 64), (2100, 32, 32, 200, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows, hq, hkv, dk, dv", CALLS)
@pytest.mark.parametrize("by_row", [False, True])
def test_outputs_lose_their_own_rounding_only(rows, hq, hkv, dk, dv, by_row):
    require_gpu()
    x = _inputs(rows, hq, hkv, dk, dv, "bf16", rows + dk, by_row=by_row, pool=3, rate=0.02)
    _check_outputs(x, [0, rows // 3, rows // 3 + 1, rows], [2, 0, 1], dk ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("rate", [2.0, 30.0])
def test_outputs_where_heads_forget_fast(rate):
    """Chunks that take exponentials of differences."""
    require_gpu()
    x = _inputs(400, 4, 2, 128, 128, "bf16", 3, pool=1, rate=rate)
    _check_outputs(x, [0, 400], [0], 0.1)


@pytest.mark.gpu
def test_a_request_answers_alike_beside_others():
    """The same tokens alone and in a call of more than 65536 rows times heads: both within the bounds of one call."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(9000, 8, 8, 128, 128, "bf16", 5, pool=2, rate=0.02)
    off = torch.tensor([0, 500, 9000], dtype=torch.int32, device="cuda")
    both = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], offsets=off)[:500]
    alone = O.decay_attention(x["q"][:500], x["k"][:500], x["v"][:500], x["log_decay"][:500])
    want, _, _ = _reference(dict({n: x[n][:500] for n in ("q", "k", "v", "log_decay")}, states=torch.zeros(1, 8, 128, 128, device="cuda")),
                            [0, 500], 128 ** -0.5, [0])
    off_by = [_norm(((y.double() - want).abs() - _half_step(want)).clamp(min=0)) / _norm(want) for y in (both, alone)]
    assert max(off_by) <= 4 * (128 + 500 + 64) ** 0.5 * E + 4 * 2.0 ** -16, off_by


@pytest.mark.gpu
@pytest.mark.parametrize("d, n", [(128, 64), (64, 60), (256, 33)])
@pytest.mark.parametrize("rate", [0.0, 0.01, 0.1])
def test_kept_states(d, n, rate):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(n, 2, 2, d, d, "bf16", n, pool=1, rate=rate)
    _, states, _ = _reference(x, [0, n], 1.0, [0])
    kept = x["states"].clone()
    O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=kept)
    err = _norm(kept.double() - states) / _norm(states)
    assert err <= ((3 * n) ** 0.5 + 8) * E, err
    assert torch.isfinite(kept).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_weights_behind_tokens_that_forget_everything(d):
    """Thirty factors of 2^-200 and then two tokens that nearly cancel: a weight is that of the decays between its tokens, which
    the sums of the chunk's decays, 6000, would leave 2^-12 of as float32."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(32, 32, 32, d, d, "bf16", d, pool=1, rate=1e-3)
    x["log_decay"][:30] = -138.0
    x["k"][31], x["v"][31] = x["k"][30], -x["v"][30]
    want, _, size = _reference(x, [0, 32], 1.0, [0])
    y = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"].clone(), scale=1.0)
    over = ((y.double() - want).abs() - _half_step(want)).clamp(min=0)
    assert (over <= ((d + 32 + 64) * E + 4 * 2.0 ** -16) * size).all(), (over / size).max()
