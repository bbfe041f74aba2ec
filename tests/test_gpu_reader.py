"""The reader on top of a network: the whole path on the GPU against the same steps in float64 on the network's output.

Bound.  The path's own roundings (8-bit and bfloat16 ones) are made in the float64 steps too.  What is left are float32
sums and roundings that fall the other way because of them or of the attention's bfloat16 exponentials: one e4m3 step in
a few hundred values, of 2^-4 each, per product, far below one bfloat16 rounding (2^-8) of every value, normwise, of
which a layer has four: 4 * 2^-8 per layer."""
import pytest

from gpu_util import require_gpu

from paper_2107_06960_amd import workloads as W


def _f8(x):
    import torch
    scale = (x.abs().amax(1) / 448).float().double()
    return (x / scale[:, None]).float().to(torch.float8_e4m3fn).double() * scale[:, None]


def _bf16(x):
    import torch
    return x.float().to(torch.bfloat16).double()


def _norm(h, gain, eps=1e-6):
    return h / (h.square().mean(1, keepdim=True) + eps).sqrt() * gain.double().cpu()


def _linear(x, p, row_adapter):
    x = _f8(x)
    y = x @ (p["w"].float().double().cpu() * p["scale"].double().cpu()[:, None]).t()
    if row_adapter is not None and p["adapters"] is not None:
        a, b, f = (t.double().cpu() for t in p["adapters"])
        for i in range(a.shape[0]):
            at = (row_adapter.cpu() == i).nonzero()[:, 0]
            y[at] += f[i] * (x[at] @ a[i].t()) @ b[i].t()
    return _bf16(y)


def _reference(params, tokens, y, hq, hkv, d, off, row_adapter):
    import torch
    frames = y.shape[0]
    kv = y.double().cpu().view(frames, -1, 2, hkv, d)
    h, delta = tokens.double().cpu(), None
    for p in params["layers"]:
        if delta is not None:
            h = _bf16(h + delta)
        q = _linear(_norm(h, p["gain"]), p["q"], row_adapter).view(-1, hq, d)
        o = torch.zeros_like(q)
        for f in range(frames):
            for j in range(hq):
                k, v = kv[f, :, 0, j // (hq // hkv)], kv[f, :, 1, j // (hq // hkv)]
                o[off[f]:off[f + 1], j] = torch.softmax(q[off[f]:off[f + 1], j] @ k.t() / d ** 0.5, -1) @ v
        delta = _linear(_norm(_bf16(o).view(len(q), -1), p["o_gain"]), p["o"], row_adapter)
    return _norm(_bf16(h + delta), params["gain"])


@pytest.mark.gpu
@pytest.mark.parametrize("rows, off, adapters", [(6, None, 0), (7, [0, 1, 7], 3), (150, [0, 140, 150], 2), (1, [0, 0, 1], 1)])
def test_reader_on_a_network(rows, off, adapters):
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import reader as R
    hq, hkv, d, width, layers = 8, 2, 64, 256, 2
    net_layers = W.YOLOV2_16 + [W.conv(2 * hkv * d, 1, act=W.LINEAR)]
    p = W.make_inputs(net_layers, 224, 192, 3, batch=2, seed=1, dtype="bf16")
    plan = M.Plan(net_layers, (224, 192, 3), "3x2/8/2x2", packed_weights=True)
    net = M.Network(plan, p, 2, "bf16")
    y = net.run(net.input_tensor(p["x"]))
    assert y.shape == (2, 14, 12, 2 * hkv * d)
    params = R.draw_params(width, hq, d, layers, seed=rows, adapters=adapters)
    reader = R.Reader(params, hq, hkv, d)
    gen = torch.Generator().manual_seed(rows)
    tokens = torch.randn(rows, width, generator=gen).bfloat16().cuda()
    offsets = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    row_adapter = torch.randint(-1, adapters, (rows,), generator=gen, dtype=torch.int32).cuda() if adapters else None
    got = reader.run(tokens, y, q_offsets=offsets, row_adapter=row_adapter)
    want = _reference(params, tokens, y, hq, hkv, d, [0, rows // 2, rows] if off is None else off, row_adapter)
    err = ((got.double().cpu() - want).norm() / want.norm()).item()
    assert err <= layers * 4 * 2.0 ** -8, err
    with pytest.raises(ValueError):
        R.Reader(params, hq, hkv, d // 2).run(tokens, y)


@pytest.mark.gpu
def test_reader_replays_on_new_frames():
    """Network and reader recorded as one graph: each replay reads the frames and tokens that are there then."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import reader as R
    hq, hkv, d, width = 4, 1, 64, 128
    net_layers = W.TINY + [W.conv(2 * hkv * d, 1, act=W.LINEAR)]
    p = W.make_inputs(net_layers, 64, 64, 3, batch=1, seed=1, dtype="bf16")
    net = M.Network(M.Plan(net_layers, (64, 64, 3), "2x2/NoCut"), p, 1, "bf16")
    reader = R.Reader(R.draw_params(width, hq, d, 1), hq, hkv, d)
    x, tokens = net.input_tensor(p["x"]), torch.randn(5, width, device="cuda").bfloat16()
    reader.run(tokens, net.run(x))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = reader.run(tokens, net.run(x))
    for seed in range(3):
        torch.manual_seed(seed)
        x.copy_(torch.rand_like(x))
        tokens.copy_(torch.randn_like(tokens))
        graph.replay()
        torch.cuda.synchronize()
        first = got.clone()
        assert torch.equal(first, reader.run(tokens, net.run(x)))
