"""Norms around a block with its gate, residual scale and residual addition (mafat_block_norm) against the formula in float64.

Bounds, from the arithmetic, with e = 2^-24: a sum of squares is a tree of float32 additions of depth below 128, so a norm's
factor is within 64 e and a few roundings of its own (its root halves the sum's error); expf and the gate's division are
within 4 e; so scale * u is within 128 e of itself and h within d = 128 e (|scale * u| + |h|).  The norm before follows h:
its factor is off by the row's d over its root mean square, and 128 e.  bfloat16 adds half a step (2^-8 of the value), e4m3
2^-4 of the value or half its smallest step, 2^-10 scales."""
import pytest

from gpu_util import require_gpu

E = 2.0 ** -24


def _tensors(rows, cols, dtype, seed, pad=0, shift=0):
    """x, gate and residual, whose rows are `cols + pad` apart and start `shift` elements into their buffer, and three gains."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def one(by):
        buf = (by * torch.randn(rows * (cols + pad) + shift, generator=g)).to(dt).cuda()
        return buf[shift:].view(rows, cols + pad)[:, :cols]

    return [one(3.0), one(2.0), one(1.0)] + [(1 + 0.3 * torch.randn(cols, generator=g)).cuda() for _ in range(3)]


def _check(args, result, f32=128 * E):
    """args: those of block_norm, in full."""
    import torch
    d = {k: v.double().cpu() if torch.is_tensor(v) else v for k, v in args.items()}
    total, y, scale = result
    u = d["x"]
    if d["after"]:
        parts = u.reshape(u.shape[0], d["groups"], -1)
        u = (parts / (parts.square().mean(-1, keepdim=True) + d["eps"]).sqrt()).reshape(u.shape)
        u = u if d["after_gain"] is None else u * d["after_gain"]
    if d["gate"] is not None:
        u = u * torch.sigmoid(d["gate"]) * (d["gate"] if d["act"] == "silu" else 1)
    u = u if d["scale"] is None else u * d["scale"]
    h = u if d["residual"] is None else u + d["residual"]
    off = f32 * (u.abs() + h.abs())
    if d["residual"] is None:
        assert total is None
    else:
        half = 2.0 ** -8 if args["x"].element_size() == 2 else 0
        assert total.dtype == args["x"].dtype
        assert ((total.double().cpu() - h).abs() <= off + half * h.abs() + 1e-38).all()
    if d["before"]:
        inv = 1 / (h.square().mean(-1, keepdim=True) + d["eps"]).sqrt()
        gain = 1 if d["before_gain"] is None else d["before_gain"]
        off = inv * abs(gain) * (off + h.abs() * (inv * off.square().mean(-1, keepdim=True).sqrt() + f32))
        h = h * inv * gain
    if args["out"] == "f8":
        most, i = h.abs().max(-1)
        s = scale.double().cpu()
        assert ((s - most / 448).abs() <= off.max(-1).values / 448 + 2 * E * s).all()
        got = y.float().double().cpu() * s[:, None]
        allowed = torch.maximum(2.0 ** -4 * h.abs(), 2.0 ** -10 * s[:, None]) * (1 + 1e-4) + 2 * off.max(-1, keepdim=True).values
        assert (y.float().abs().amax(-1) == 448).all()
    else:
        assert scale is None
        got, allowed = y.double().cpu(), off + (2.0 ** -8 * h.abs() if args["out"] == "bf16" else 0) + 1e-38
    assert ((got - h).abs() <= allowed).all()


def _run(x, gate, residual, a, s, b, **kw):
    from paper_2107_06960_amd import operators as O
    args = dict(x=x, after=True, after_gain=a, groups=1, gate=gate, act="silu", scale=s, residual=residual, before=True,
                before_gain=b, eps=1e-5, out="f8")
    args.update(kw)
    _check(args, O.block_norm(**args))


# columns, groups: every number of pieces per thread and team size, the lengths around them; parts of lanes, of pieces, of
# values that no piece ends with; rows read again
SIZES = [(1, 1), (3, 1), (64, 1), (127, 1), (128, 1), (129, 1), (511, 1), (520, 1), (1001, 1), (1024, 1), (1031, 1), (2048, 1),
         (2056, 1), (4096, 1), (4097, 1), (8192, 1), (8200, 1), (16384, 1), (16385, 1), (40001, 1),
         (64, 8), (64, 4), (512, 8), (2048, 16), (4096, 32), (8192, 64), (16384, 128), (1024, 2), (4096, 2), (96, 4), (240, 3), (960, 5),
         (3200, 25), (9600, 3), (16320, 20), (33, 3), (40, 40), (1001, 7), (1000, 8), (40000, 10), (4096, 4096), (6000, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols, groups", SIZES)
def test_block_norm_against_the_formula(cols, groups, dtype):
    require_gpu()
    rows = 5 if cols > 2048 else 19
    t = _tensors(rows, cols, dtype, cols + groups)
    _run(*t, groups=groups)
    _run(*t, groups=groups, out=dtype, act="sigmoid")
    x, gate, res, a, s, b = t
    _run(x, gate, None, a, None, None, groups=groups, before=False, out="f8")
    _run(x, None, res, None, s, b, groups=groups, out="bf16")
    _run(x, None, res, None, None, b, groups=groups, after=False, out="f32")
    _run(x, gate, None, None, None, None, groups=groups, after=False, before=False, out=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols, groups, pad, shift", [(256, 4, 8, 0), (250, 2, 7, 1), (1001, 1, 23, 3), (4096, 16, 1, 5), (33000, 3, 5, 1)])
def test_strided_and_unaligned_rows(cols, groups, pad, shift, dtype):
    require_gpu()
    for out in ("f8", dtype):
        _run(*_tensors(7, cols, dtype, cols + pad, pad, shift), groups=groups, out=out)


@pytest.mark.gpu
def test_many_rows_and_one():
    require_gpu()
    from paper_2107_06960_amd import operators as O
    for rows, cols in [(1, 1024), (1, 4096), (16411, 40), (3001, 256), (777, 4096)]:
        _run(*_tensors(rows, cols, "bf16", rows))
    x, gate, res, a, s, b = _tensors(1, 64, "bf16", 1)
    h, y, scale = O.block_norm(x[:0], residual=res[:0])
    assert h.shape == y.shape == (0, 64) and scale.shape == (0,)


@pytest.mark.gpu
@pytest.mark.parametrize("cols, groups", [(64, 1), (1000, 1), (4096, 1), (36000, 1), (512, 8), (960, 5), (1001, 7)])
def test_rows_of_zeros_nan_and_infinities_stay_theirs(cols, groups):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, gate, res, a, s, b = _tensors(8, cols, "f32", cols)

    def run(out="f8"):
        return O.block_norm(x, after_gain=a, groups=groups, gate=gate, scale=s, residual=res, before_gain=b, out=out)

    clean = run()
    x[1], res[1] = 0, 0
    x[3, cols // 2] = float("nan")
    x[5, cols - 1] = float("inf")
    res[6, 0] = float("-inf")
    gate[2, 3] = float("nan")
    h, y, scale = run()
    yf = y.float()
    assert torch.equal(yf[1], torch.zeros_like(yf[1])) and scale[1] == 1
    for row in (2, 3, 5, 6):
        assert torch.isnan(scale[row]) and torch.isnan(yf[row]).any()
    for row in (0, 4, 7):  # the others do not change
        assert torch.equal(yf[row], clean[1].float()[row]) and scale[row] == clean[2][row] and torch.equal(h[row], clean[0][row])
    assert torch.isnan(run("f32")[1][3]).all()


@pytest.mark.gpu
def test_gates_far_out():
    """act saturates: no overflow where exp(-gate) does."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    gate = torch.tensor([[-1e4, -200.0, -80.0, 0.0, 80.0, 200.0, 1e4, 3e38]], device="cuda")
    x = torch.full_like(gate, 2.0)
    for act in ("silu", "sigmoid"):
        _, y, _ = O.block_norm(x, after=False, gate=gate, act=act, before=False, out="f32")
        want = 2 * torch.sigmoid(gate.double()) * (gate.double() if act == "silu" else 1)
        # (2 * 3e38 is past float32: the value that it stands for there is infinity)
        assert ((y == want.float()) | ((y.double() - want).abs() <= 8 * E * want.abs() + 1e-36)).all(), y


@pytest.mark.gpu
def test_eps_in_a_tensor_is_read_at_every_call():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, _, res, a, s, b = _tensors(3, 64, "f32", 5)
    eps = torch.tensor(1e-6)
    for value in (1e-6, 0.5, 1e-6):
        eps.fill_(value)
        got = O.block_norm(x, eps=eps, out="f32")[1]
        assert torch.equal(got, O.block_norm(x, eps=eps.item(), out="f32")[1])
    assert not torch.equal(got, O.block_norm(x, eps=0.5, out="f32")[1])


@pytest.mark.gpu
def test_python_refusals():
    require_gpu()
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    x, gate, res, a, s, b = _tensors(4, 64, "bf16", 1)
    for args, kw in [((x.half(),), {}), ((x.cpu(),), {}), ((x[0],), {}), ((x.t(),), {}), ((x,), {"gate": gate[:3]}),
                     ((x,), {"gate": gate.float()}), ((x,), {"residual": res[:, :63]}), ((x,), {"after_gain": a.bfloat16()}),
                     ((x,), {"scale": s[:63]}), ((x,), {"before_gain": b.cpu()}), ((x,), {"act": "gelu"}), ((x,), {"out": "f16"}),
                     ((x[:1].expand(4, 64),), {})]:
        with pytest.raises(ValueError):
            O.block_norm(*args, **kw)
    for kw in ({"eps": -1.0}, {"groups": 3}, {"groups": 0}, {"after": False, "after_gain": a}, {"before": False, "before_gain": b}):
        with pytest.raises(M.MafatError):
            O.block_norm(x, **kw)
    with pytest.raises(ValueError, match="forward only"):
        O.block_norm(x, after_gain=a.requires_grad_())


@pytest.mark.gpu
def test_runs_on_the_current_stream_and_replays():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    x, gate, res, a, s, b = _tensors(9, 768, "bf16", 3)

    def run():
        return O.block_norm(x, after_gain=a, groups=6, gate=gate, scale=s, residual=res, before_gain=b)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        x.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, run()):
            assert torch.equal(g.float(), w.float())
