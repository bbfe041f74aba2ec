"""Linear attention with decays (mafat_decay_attention) against the recurrence in float64, token after token.

Bounds.  In float32 (e = 2^-24) a state is a sum over tokens and an output one over tokens and key entries, of terms with a few
roundings each and an exponent that is off by e times its size (a term 2^-c is off by c ln 2 e of itself, largest where
c 2^-c is, 0.54); n such roundings in any order stay below n e of the sum of magnitudes, and add up like sqrt(n) where they
are independent.  So singly: (dk + n + 64) e of the sums of magnitudes, n the tokens; as a whole: the norm of the error
below 4 sqrt(dk + n + 64) e of the norm of what the sums of magnitudes would be if signs did not cancel at all, which for
random signs is the norm of the value itself.  bfloat16 outputs add their own rounding, 2^-8, and the kernel for whole tiles
rounds scores, and in large calls the states that rows read, to bfloat16, again 2^-8 each as independent errors: three roundings of 2^-8
bound the outputs as a whole.  Its states stay within 2^-16: weighted values enter them in parts that leave 2^-17 of a term
or less."""
import math

import pytest

from gpu_util import require_gpu

E = 2.0 ** -24


def _reference(q, k, v, log_decay, states, slots, off, scale):
    """(y, states after, y and states with every term's magnitude) in float64 on the CPU."""
    import torch
    q, k, v, g = (t.double().cpu() for t in (q, k, v, log_decay))
    g = g.clamp(max=0)
    rows, hq, dk = q.shape
    hkv, dv = k.shape[1], v.shape[2]
    y, ya = torch.zeros(rows, hq, dv, dtype=torch.float64), torch.zeros(rows, hq, dv, dtype=torch.float64)
    pool = None if states is None else states.double().cpu().clone()
    pool_a = None if states is None else pool.abs()
    seen = set()
    for r in range(len(off) - 1):
        lo, hi = (min(max(o, 0), rows) for o in off[r:r + 2])
        if hi <= lo:
            continue
        slot = -1 if pool is None else r if slots is None else slots[r]
        slot = slot if pool is not None and 0 <= slot < pool.shape[0] else -1
        if slot in seen:
            y[lo:hi] = math.nan
            continue
        s = torch.zeros(hkv, dk, dv, dtype=torch.float64) if slot < 0 else pool[slot].clone()
        sa = s.abs()
        for t in range(lo, hi):
            a = (g[t] if g.dim() == 2 else g).exp()[:, None, None]
            kv = k[t][:, :, None] * v[t][:, None, :]
            s, sa = a * s + kv, a * sa + kv.abs()
            qt = q[t].view(hkv, -1, dk)
            y[t] = scale * (qt @ s).view(hq, dv)
            ya[t] = abs(scale) * (qt.abs() @ sa).view(hq, dv)
        if slot >= 0:
            seen.add(slot)
            pool[slot], pool_a[slot] = s, sa
    return y, pool, ya, pool_a


def _inputs(rows, hq, hkv, dk, dv, dtype, seed, by_row=True, pool=0, rate=0.1):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(shape, generator=gen)

    g = -rate * (randn(rows, hkv) if by_row else randn(hkv)).exp()
    return dict(q=randn(rows, hq, dk).to(dt).cuda(), k=randn(rows, hkv, dk).to(dt).cuda(), v=randn(rows, hkv, dv).to(dt).cuda(),
                log_decay=g.cuda(), states=2 * randn(pool, hkv, dk, dv).cuda() if pool else None)


def _norm(t):
    return t.norm().item()


def _check(x, off=None, slots=None, scale=None, requests=None, rows_of_none=()):
    """Runs and checks every row that a request has, and every state."""
    import torch
    from paper_2107_06960_amd import operators as O
    rows, _, dk = x["q"].shape
    scale = dk ** -0.5 if scale is None else scale
    n = requests if requests is not None else len(off) - 1 if off is not None else len(slots) if slots is not None else (
        x["states"].shape[0] if x["states"] is not None else 1)
    cuts = [i * (rows // n) for i in range(n + 1)] if off is None else off
    want, states, size, sizes = _reference(x["q"], x["k"], x["v"], x["log_decay"], x["states"], slots, cuts, scale)
    kept = None if x["states"] is None else x["states"].clone()

    def ints(v):
        return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")

    y = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=kept, slots=ints(slots), offsets=ints(off), scale=scale)
    assert y.dtype == x["q"].dtype and y.shape == want.shape
    mine = torch.zeros(rows, dtype=torch.bool)
    for a, b in zip(cuts, cuts[1:]):
        mine[max(a, 0):max(min(b, rows), 0)] = True
    got, want, size = y.double().cpu()[mine], want[mine], size[mine]
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    got, want, size = got[fine], want[fine], size[fine]
    most = max([b - a for a, b in zip(cuts, cuts[1:])] + [1])
    each, whole = (dk + most + 64) * E, 4 * (dk + most + 64) ** 0.5 * E
    bf16 = x["q"].element_size() == 2
    err = (got - want).abs()
    assert (err <= each * size + (2.0 ** -8 * want.abs() + 2.0 ** -8 * size if bf16 else 0) + 1e-37).all(), (err / size).max()
    assert _norm(err) <= (whole + (3 * 2.0 ** -8 if bf16 else 0)) * _norm(want) + 1e-30, _norm(err) / _norm(want)
    if kept is not None:
        err = (kept.double().cpu() - states).abs()
        assert (err <= (each + (2.0 ** -16 if bf16 else 0)) * sizes + 1e-37).all(), (err / sizes).max()
        assert _norm(err) <= (whole + (2.0 ** -16 if bf16 else 0)) * _norm(states) + 1e-30, _norm(err) / _norm(states)
    return y, kept


DIMS = [(64, 64), (128, 128), (128, 64), (64, 128), (256, 256), (80, 48), (1, 1), (3, 200), (37, 65), (200, 16), (96, 96), (32, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk, dv", DIMS)
def test_single_tokens(dk, dv, dtype):
    require_gpu()
    for requests, hq, hkv in [(1, 1, 1), (3, 4, 2), (70, 3, 3)]:
        _check(_inputs(requests, hq, hkv, dk, dv, dtype, dk + dv, by_row=requests != 3, pool=requests))
    # two tokens each, some with one, none, three; the states elsewhere in the pool
    _check(_inputs(8, 4, 2, dk, dv, dtype, dk, pool=7), off=[0, 1, 1, 3, 6, 8], slots=[6, 2, 0, 5, 1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk, dv", DIMS)
def test_prompts(dk, dv, dtype):
    require_gpu()
    _check(_inputs(45, 2, 1, dk, dv, dtype, dk + 2 * dv, pool=1))
    _check(_inputs(130, 3, 3, dk, dv, dtype, dk + 3 * dv, by_row=False, pool=4), off=[0, 1, 65, 65, 130], slots=[3, 1, 0, 2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 255, 256, 257, 320, 321, 511, 513])
def test_lengths_around_chunks_and_segments(n, dtype):
    require_gpu()
    _check(_inputs(n, 2, 1, 64, 64, dtype, n, pool=1))
    _check(_inputs(n + 300, 2, 2, 64, 32, dtype, n, by_row=False, pool=2), off=[0, n, n + 300], slots=[1, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk, dv, hq, hkv", [(128, 128, 2, 2), (64, 64, 4, 1), (80, 48, 2, 1), (64, 256, 1, 1)])
def test_segments(dk, dv, hq, hkv, dtype):
    """Requests of several segments beside short, empty and single-token ones."""
    require_gpu()
    off = [0, 700, 701, 701, 1500, 1530, 2048]
    x = _inputs(2048, hq, hkv, dk, dv, dtype, dk, pool=8, rate=0.01)
    _check(x, off=off, slots=[5, 2, 0, 7, 1, 3])
    _check(dict(x, states=None), off=off)
    _check(_inputs(1200, hq, hkv, dk, dv, dtype, dv, by_row=False, pool=2, rate=0.003))
    # a state that is not kept, one that two requests name, one that an empty request names first
    _check(x, off=off, slots=[5, 8, 7, -1, 5, 7])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_and_the_same_slot(dtype):
    """More requests than a wave has lanes, some with a state that an earlier one has."""
    require_gpu()
    import random
    r = random.Random(1)
    for rows in (400, 150):
        off = sorted(r.randint(0, rows) for _ in range(149))
        slots = [r.randrange(-1, 200) for _ in range(150)]
        x = _inputs(rows, 2, 1, 32, 32, dtype, 7, pool=199)
        _check(x, off=[0] + off + [rows], slots=slots)


@pytest.mark.gpu
@pytest.mark.parametrize("rows, heads", [(4100, 16), (9000, 8)])
def test_large_calls(rows, heads):
    """Above 65536 rows times heads the states that rows read are rounded once."""
    require_gpu()
    _check(_inputs(rows, heads, heads, 32, 32, "bf16", rows, pool=2, rate=0.01), off=[0, rows // 3, rows])


@pytest.mark.gpu
def test_a_slot_that_a_request_far_before_has():
    """Past the first 64 requests and the 512 after them."""
    require_gpu()
    x = _inputs(1400, 1, 1, 16, 16, "f32", 11, pool=1400)
    slots = list(range(1400))
    for later, earlier in ((63, 0), (64, 63), (65, 64), (575, 64), (576, 575), (577, 0), (1399, 576), (1398, 1100), (1000, 999)):
        slots[later] = slots[earlier]
    _check(x, slots=slots)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 40, 600])
def test_rows_behind_the_last_request_stay(rows, dtype):
    require_gpu()
    import ctypes
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    x = _inputs(rows + 50, 2, 1, 64, 64, dtype, rows, pool=2)
    off = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    want = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"].clone(), offsets=off)
    # into rows and heads with gaps, which stay as well
    y = torch.full((rows + 50, 2, 80), 7.0, dtype=x["q"].dtype, device="cuda")
    c = O.mafat_decay(M.MAFAT_BF16 if dtype == "bf16" else M.MAFAT_F32, 2, rows + 50, 2, 2, 1, 64, 64, 0.125, 1, 128, 64, 64, 64, 64, 64,
                      160, 80, 1, 64 * 64)
    need = O.mafat_decay_workspace(c)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")  # NaNs: nothing of it is read before it is written
    states = x["states"].clone()
    O.mafat_decay_attention(c, x["q"].data_ptr(), x["k"].data_ptr(), x["v"].data_ptr(), x["log_decay"].data_ptr(), off.data_ptr(),
                            states.data_ptr(), None, y.data_ptr(), ws.data_ptr() if need else None, need, M._stream_handle(None))
    torch.cuda.synchronize()
    assert torch.equal(y[:rows, :, :64], want[:rows])
    assert (y[rows:] == 7).all() and (y[:, :, 64:] == 7).all()
    assert ctypes.sizeof(c) and torch.isfinite(states).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, shift, pad", [(64, 0, 8), (128, 1, 0), (64, 4, 3), (48, 3, 5)])
def test_strided_and_unaligned(d, shift, pad, dtype):
    """q, k and v side by side in the rows of one projection; states with gaps between them."""
    require_gpu()
    import torch
    for rows, requests in ((90, 2), (4, 4), (700, 1)):
        x = _inputs(rows, 4, 2, d, d, dtype, d + rows, pool=requests)
        buf = torch.zeros(rows * (8 * d + pad) + shift, dtype=x["q"].dtype, device="cuda")
        row = buf[shift:].view(rows, 8 * d + pad)
        parts = [row[:, :4 * d].view(rows, 4, d), row[:, 4 * d:6 * d].view(rows, 2, d), row[:, 6 * d:8 * d].view(rows, 2, d)]
        for p, n in zip(parts, "qkv"):
            p.copy_(x[n])
        wide = torch.zeros(requests, 2 * d * d + 5, device="cuda")
        wide[:, :2 * d * d] = x["states"].view(requests, -1)
        wide_g = torch.zeros(rows, 7, device="cuda")
        wide_g[:, :2] = x["log_decay"]
        want, kept = _check(x)
        from paper_2107_06960_amd import operators as O
        states = wide[:, :2 * d * d].view(requests, 2, d, d)
        y = O.decay_attention(*parts, wide_g[:, :2], states=states)
        bf16 = dtype == "bf16"
        assert _norm((y - want).double()) <= (3 * 2.0 ** -8 if bf16 else 2.0 ** -18) * _norm(want.double())
        assert _norm((states - kept).double()) <= 2.0 ** -15 * _norm(kept.double())
        assert (wide[:, 2 * d * d:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 70, 600])
def test_decays_at_their_ends(n, dtype):
    """No decay, decays that forget at once (minus infinity among them), above 0."""
    require_gpu()
    import torch
    x = _inputs(n, 2, 2, 64, 64, dtype, n, pool=1)
    for kind in range(4):
        g = x["log_decay"].clone()
        if kind == 0:
            g.zero_()
        elif kind == 1:
            g[::3] = -math.inf
            g[1::5] = -1e30
        elif kind == 2:
            g[::2] = 5.0
        else:
            g.mul_(200)
        _check(dict(x, log_decay=g))
    g = torch.tensor([0.0, -math.inf], device="cuda")
    _check(dict(x, log_decay=g))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, at", [(2, 1), (40, 17), (100, 70), (700, 300), (700, 620)])
@pytest.mark.parametrize("where, value", [("q", math.nan), ("k", math.inf), ("v", math.nan), ("v", -math.inf), ("log_decay", math.nan)])
def test_what_is_not_finite_reaches_later_rows_of_its_request_only(n, at, where, value, dtype):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(2 * n, 2, 1, 64, 64, dtype, n, pool=2, rate=0.01)

    def run():
        states = x["states"].clone()
        return O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=states), states

    clean, clean_states = run()
    x[where].view(2 * n, -1)[at, 0] = value
    y, states = run()
    assert torch.isfinite(y[:at]).all() and not torch.isfinite(y[at]).all()
    tight = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -18  # (the chunk may have been summed in another order)
    assert _norm((y[:at] - clean[:at]).double()) <= tight * _norm(clean[:at].double())
    assert torch.equal(y[n:], clean[n:]) and torch.equal(states[1], clean_states[1])
    if where == "q":
        assert torch.equal(states, clean_states) and torch.equal(y[at + 1:], clean[at + 1:])
    else:
        assert not torch.isfinite(states[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rate", [2.0, 30.0])
def test_what_is_not_finite_where_heads_forget_fast(rate, dtype):
    """Chunks that forget more than their sums are kept for, with values that are not finite in the middle."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(500, 4, 2, 64, 64, dtype, 9, pool=1, rate=rate)
    clean, _ = _check(x)
    x["v"][333, 1, 7] = math.nan
    x["v"][340, 1, 9] = math.inf
    y = O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"].clone())
    other = torch.ones_like(y, dtype=torch.bool)
    other[333:, 2:, 7] = False
    other[340:, 2:, 9] = False
    tight = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -18
    assert torch.isfinite(y[other]).all() and torch.isnan(y[333, 2:, 7]).all() and not torch.isfinite(y[340, 2:, 9]).any()
    assert _norm((y[other] - clean[other]).double()) <= tight * _norm(clean[other].double())


@pytest.mark.gpu
def test_offsets_that_decrease_stay_inside():
    """Which rows are computed is open then, but nothing outside of the tensors is touched, and what follows is right."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(700, 2, 1, 64, 64, "bf16", 3, pool=4)
    for off in ([0, 700, 0, 700, 0], [700, 0, 350, 100, 700], [-5, 2000, -7, 300, 1 << 30]):
        O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"].clone(),
                          offsets=torch.tensor(off, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    _check(x, off=[0, 300, 300, 650, 700])


@pytest.mark.gpu
def test_chunks_and_single_tokens_agree():
    """A prompt at once, in two calls, and its last tokens one by one."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(300, 4, 2, 64, 64, "f32", 5, pool=1)

    def part(a, b, states):
        return O.decay_attention(x["q"][a:b], x["k"][a:b], x["v"][a:b], x["log_decay"][a:b], states=states)

    one, many = x["states"].clone(), x["states"].clone()
    whole = part(0, 300, one)
    parts = torch.cat([part(a, b, many) for a, b in [(0, 200), (200, 290)] + [(i, i + 1) for i in range(290, 300)]])
    for got, want in ((parts, whole), (many, one)):
        assert _norm((got - want).double()) <= 8 * (64 + 300) ** 0.5 * E * _norm(want.double())


@pytest.mark.gpu
def test_nothing_to_do():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x = _inputs(5, 2, 1, 32, 32, "bf16", 1, pool=3)
    before = x["states"].clone()
    y = O.decay_attention(x["q"][:0], x["k"][:0], x["v"][:0], x["log_decay"][:0], states=x["states"],
                          offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert y.shape == (0, 2, 32) and torch.equal(x["states"], before)
    O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"], offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert torch.equal(x["states"], before)
    _check(dict(x, states=torch.empty(0, 1, 32, 32, device="cuda")), off=[0, 2, 5])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 100, 700])
def test_replays_two_graphs_and_another_stream(n):
    """Two graphs of their own workspaces, replayed in turn, on states that go on."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    xs = [_inputs(2 * n, 2, 1, 64, 64, "bf16", s, pool=2) for s in (1, 2)]

    def run(x):
        return O.decay_attention(x["q"], x["k"], x["v"], x["log_decay"], states=x["states"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(dict(xs[0], states=xs[0]["states"].clone()))
    torch.cuda.synchronize()
    first = [x["states"].clone() for x in xs]
    graphs, got = [], []
    for x in xs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(run(x))
        graphs.append(graph)
    for x, s in zip(xs, first):
        x["states"].copy_(s)
    for i in range(3):
        before = [x["states"].clone() for x in xs]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, s, y in zip(xs, before, got):
            assert torch.equal(run(dict(x, states=s)), y) and torch.equal(s, x["states"])
        xs[i % 2]["q"].mul_(-0.5)


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    x = _inputs(6, 4, 2, 64, 32, "bf16", 1, pool=3)
    q, k, v, g, s = (x[n] for n in ("q", "k", "v", "log_decay", "states"))
    i32 = dict(dtype=torch.int32, device="cuda")
    for args, kw in [((q.half(), k, v, g), {}), ((q.cpu(), k, v, g), {}), ((q[0], k, v, g), {}), ((q, k[:5], v, g), {}),
                     ((q, k.float(), v, g), {}), ((q, k[..., :32], v, g), {}), ((q, k, v[:, :1], g), {}), ((q, k, v.float(), g), {}),
                     ((q, k, v, g.bfloat16()), {}), ((q, k, v, g[:5]), {}), ((q, k, v, g[:, :1]), {}), ((q, k, v, g.cpu()), {}),
                     ((q[:, :3], k, v, g), {}), ((q, k, v, g.t().contiguous().t()), {}), ((q, k, v, g), {"states": s.half()}),
                     ((q, k, v, g), {"states": s[:, :1]}), ((q, k, v, g), {"states": s.transpose(2, 3)}),
                     ((q, k, v, g), {"states": s.transpose(2, 3).contiguous().transpose(2, 3)}),
                     ((q, k, v, g), {"slots": torch.zeros(1, **i32)}), ((q, k, v, g), {"states": s, "slots": torch.zeros(3, device="cuda")}),
                     ((q, k, v, g), {"states": s, "slots": torch.zeros(3, **i32), "offsets": torch.zeros(3, **i32)}),
                     ((q, k, v, g), {"offsets": torch.zeros(1, **i32)}), ((q.transpose(1, 2).contiguous().transpose(1, 2), k, v, g), {})]:
        with pytest.raises(ValueError):
            O.decay_attention(*args, **kw)
    for kw in ({"scale": math.nan}, {"states": s[:1].expand(3, 2, 64, 32)}, {"states": torch.zeros(4, 2, 64, 32, device="cuda")}):
        with pytest.raises(M.MafatError):
            O.decay_attention(q, k, v, g, **kw)
    with pytest.raises(M.MafatError):
        O.decay_attention(torch.zeros(2, 1, 300, device="cuda"), torch.zeros(2, 1, 300, device="cuda"), torch.zeros(2, 1, 8, device="cuda"),
                          torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError, match="forward only"):
        O.decay_attention(q, k, v, g, states=s.requires_grad_())
