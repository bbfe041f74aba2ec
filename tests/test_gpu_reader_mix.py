"""A reader whose layers mix the tokens of each request: rotary positions, linear attention with decays and the norms around
the block together, as they are used, against the same steps in float64.

Bound.  The path's own roundings to 8 bits and bfloat16 are made in the float64 steps too; what is left are roundings that
fall the other way (see test_gpu_reader.py: four of bfloat16 a layer, 2^-8 each, normwise) and, in a mixing layer, the
projection, the turned queries and keys, linear attention's three (its scores, the states that rows read and its output) and
the two sums after it: eleven of 2^-8 a layer.  States are float32 sums over keys and values whose own last bits may differ:
two roundings of 2^-8, and what the layers before add."""
import pytest

from gpu_util import require_gpu
from test_gpu_reader import _bf16, _f8, _linear, _norm

from paper_2107_06960_amd import workloads as W


def _turned(x, positions):
    import math
    import torch
    half = x.shape[-1] // 2
    t = positions.double()[:, None, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    a, b = x[..., :half], x[..., half:]
    return _bf16(torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], -1))


def _mixed(p, h, next_gain, heads, dim, positions, off, states, slots):
    """(sum, its norm) of the layer's mixing; states: [slots, heads, dim, dim] float64, updated."""
    import torch
    rows, n = h.shape[0], heads * dim
    all_ = _linear(_norm(h, p["gain"]), p["qkvg"], None)
    q, k, v = (all_[:, i * n:(i + 1) * n].view(rows, heads, dim) for i in range(3))
    q, k = _turned(q, positions), _turned(k, positions)
    a = p["log_decay"].double().cpu().exp()[:, None, None]
    o = torch.zeros(rows, heads, dim, dtype=torch.float64)
    for r in range(len(off) - 1):
        s = states[slots[r]]
        for t in range(off[r], off[r + 1]):
            s = a * s + k[t][:, :, None] * v[t][:, None, :]
            o[t] = (q[t][:, None] @ s)[:, 0] / dim ** 0.5
        states[slots[r]] = s
    o = _bf16(o)
    u = o / (o.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    g = all_[:, 3 * n:]
    u = u.reshape(rows, n) * p["o_gain"].double().cpu() * g * torch.sigmoid(g)
    delta = _linear(u, p["o"], None)
    h = h + _norm(delta, p["after_gain"]) * p["scale"].double().cpu()
    return _bf16(h), _norm(h, next_gain)


def _reference(params, tokens, y, hq, hkv, d, q_off, heads, dim, positions, off, memory, slots):
    import torch
    kv = y.double().cpu().view(y.shape[0], -1, 2, hkv, d)
    h, delta = tokens.double().cpu(), None
    for i, p in enumerate(params["layers"]):
        if delta is not None:
            h = _bf16(h + delta)
        h, x = _mixed(p["mix"], h, p["gain"], heads, dim, positions.cpu(), off, memory[i], slots)
        q = _linear(x, p["q"], None).view(-1, hq, d)
        o = torch.zeros_like(q)
        for f in range(y.shape[0]):
            for j in range(hq):
                k, v = kv[f, :, 0, j // (hq // hkv)], kv[f, :, 1, j // (hq // hkv)]
                o[q_off[f]:q_off[f + 1], j] = torch.softmax(q[q_off[f]:q_off[f + 1], j] @ k.t() / d ** 0.5, -1) @ v
        delta = _linear(_norm(_bf16(o).view(len(q), -1), p["o_gain"]), p["o"], None)
    return _norm(_bf16(h + delta), params["gain"])


HQ, HKV, D, WIDTH, HEADS, DIM = 4, 2, 64, 256, 3, 64


def _setup(layers=2):
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import reader as R
    net_layers = W.TINY + [W.conv(2 * HKV * D, 1, act=W.LINEAR)]
    p = W.make_inputs(net_layers, 64, 64, 3, batch=2, seed=1, dtype="bf16")
    net = M.Network(M.Plan(net_layers, (64, 64, 3), "2x2/NoCut"), p, 2, "bf16")
    params = R.draw_params(WIDTH, HQ, D, layers, seed=2, mix_heads=HEADS, mix_dim=DIM)
    return net, net.input_tensor(p["x"]), params, R.Reader(params, HQ, HKV, D, mix_heads=HEADS, mix_dim=DIM)


def _ints(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [[1, 1], [5, 0, 70], [130, 33, 1], [3]])
def test_prompts_then_single_tokens(lengths):
    require_gpu()
    import torch
    layers = 2
    net, image, params, reader = _setup(layers)
    y = net.run(image)
    requests, slots = len(lengths), [4, 1, 2][:len(lengths)]
    off = [sum(lengths[:i]) for i in range(requests + 1)]
    gen = torch.Generator().manual_seed(off[-1])
    memory = reader.memory(6)
    memory.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    want_memory = memory.double().cpu()
    before = want_memory.clone()
    bound = layers * 11 * 2.0 ** -8
    start = [10 * i for i in range(requests)]
    for step in range(3):  # the prompts, then a token of each request twice
        n = lengths if step == 0 else [1] * requests
        off = [sum(n[:i]) for i in range(requests + 1)]
        rows = off[-1]
        q_off = [0, off[1], rows]  # request 0 is about frame 0, the others about frame 1
        tokens = torch.randn(rows, WIDTH, generator=gen).bfloat16().cuda()
        positions = _ints([start[r] + i for r in range(requests) for i in range(n[r])])
        start = [s + m for s, m in zip(start, n)]
        got = reader.run(tokens, y, q_offsets=_ints(q_off), positions=positions, offsets=_ints(off), memory=memory, slots=_ints(slots))
        want = _reference(params, tokens, y, HQ, HKV, D, q_off, HEADS, DIM, positions, off, want_memory, slots)
        err = ((got.double().cpu() - want).norm() / want.norm()).item()
        assert err <= bound, (step, err)
        err = ((memory.double().cpu() - want_memory).norm() / want_memory.norm()).item()
        assert err <= bound, (step, err)
    rest = [i for i in range(6) if i not in slots]
    assert torch.equal(memory.double().cpu()[:, rest], before[:, rest])  # places that no request names


@pytest.mark.gpu
def test_decode_steps_replay():
    """Network and reader as one graph: each replay reads the tokens and positions that are there then, and goes on from the
    memory that the last one left."""
    require_gpu()
    import torch
    net, image, params, reader = _setup(1)
    tokens, positions = torch.randn(4, WIDTH, device="cuda").bfloat16(), _ints([7, 3, 0, 100])
    memory, again = reader.memory(4), reader.memory(4)
    reader.run(tokens, net.run(image), positions=positions, memory=reader.memory(4), slots=_ints([3, 0, 1, 2]))
    slots = _ints([3, 0, 1, 2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = reader.run(tokens, net.run(image), positions=positions, memory=memory, slots=slots)
    memory.zero_()
    for seed in range(3):
        torch.manual_seed(seed)
        tokens.copy_(torch.randn_like(tokens))
        positions.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, reader.run(tokens, net.run(image), positions=positions, memory=again, slots=slots))
        assert torch.equal(memory, again) and memory.abs().sum() > 0


def test_refusals():
    import torch
    from paper_2107_06960_amd import reader as R
    tokens, maps = torch.zeros(2, 64), torch.zeros(1, 2, 2, 64)
    plain = R.Reader(R.draw_params(64, 2, 32, 1, device="cpu"), 2, 1, 32)
    for kw in ("positions", "offsets", "memory", "slots"):
        with pytest.raises(ValueError, match="no layer does"):
            plain.run(tokens, maps, **{kw: torch.zeros(2, dtype=torch.int32)})
    mixing = R.draw_params(64, 2, 32, 1, device="cpu", mix_heads=2, mix_dim=16)
    with pytest.raises(ValueError, match="positions"):
        R.Reader(mixing, 2, 1, 32, mix_heads=2, mix_dim=16).run(tokens, maps)
    with pytest.raises(ValueError, match="mix_heads"):
        R.Reader(mixing, 2, 1, 32).run(tokens, maps, positions=torch.zeros(2, dtype=torch.int32))
