"""Operators among a reader's tokens on tensors past 2^31 elements and at odd addresses: the same bits as on small copies of
what they read."""
import pytest

from gpu_util import require_gpu


def _far(rows, width, row, dtype, seed):
    """[rows, width] with `row` elements between rows, and a contiguous copy."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.empty(rows * row, dtype=dtype, device="cuda")
    x = buf.view(rows, row)[:, :width]
    x.copy_(torch.randn(rows, width, generator=gen, device="cuda"))
    return x, x.contiguous()


@pytest.mark.gpu
def test_rows_past_2_31_elements():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    rows, row = 40000, 1 << 16
    x, near = _far(rows, 3 * 128, row, torch.bfloat16, 1)
    assert (rows - 1) * row > 2 ** 31
    positions, turns = torch.arange(rows, dtype=torch.int32, device="cuda"), O.rotary_turns(32)
    for got, want in zip(*(O.rotary(t[:, :256].unflatten(1, (2, 128)), positions, turns, k=t[:, 256:].unflatten(1, (1, 128)))
                           for t in (x, near))):
        assert torch.equal(got, want)
    for got, want in zip(*(O.block_norm(t[:, :128], gate=t[:, 128:256], residual=t[:, 256:]) for t in (x, near))):
        assert torch.equal(got.float(), want.float())
    decay = torch.full((2,), -0.01, device="cuda")
    for dk in (64, 60):  # whole pieces, and the kernel for any size
        outs = []
        for t in (x, near):
            q, k, v = (t[:, 128 * i:128 * i + 2 * dk].unflatten(1, (2, dk)) for i in range(3))
            states = torch.zeros(2, 2, dk, dk, device="cuda")  # two requests of 20000 rows
            outs.append((O.decay_attention(q, k, v, decay, states=states), states))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 90])
def test_states_past_2_31_elements(rows):
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    slots, d = (1 << 31) // (64 * 64) + 8, 64
    gen = torch.Generator(device="cuda").manual_seed(rows)
    pool = torch.empty(slots, 1, d, d, device="cuda")
    at = torch.tensor([slots - 1, 3], dtype=torch.int32, device="cuda")
    pool[at.long()] = torch.randn(2, 1, d, d, generator=gen, device="cuda")
    q, k, v = (torch.randn(rows, 1, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    decay = torch.full((1,), -0.1, device="cuda")
    small = pool[at.long()].clone()
    want = O.decay_attention(q, k, v, decay, states=small)
    got = O.decay_attention(q, k, v, decay, states=pool, slots=at)
    assert torch.equal(got, want) and torch.equal(pool[at.long()], small)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 90, 700])
def test_outputs_at_odd_addresses(rows):
    """Rows and heads of y at any element, with what lies between them left as it was."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import mafat as M
    from paper_2107_06960_amd import operators as O
    d, head, row = 64, 67, 2 * 67 + 1
    gen = torch.Generator(device="cuda").manual_seed(rows)
    q, k, v = (torch.randn(rows, 2, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    decay = torch.full((2,), -0.02, device="cuda")
    states = torch.zeros(1, 2, d, d, device="cuda")
    want = O.decay_attention(q, k, v, decay, states=states.clone())
    buf = torch.full((rows * row + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    c = O.mafat_decay(M.MAFAT_BF16, 1, rows, 1, 2, 2, d, d, d ** -0.5, 0, *[2 * d, d] * 3, row, head, 2, 2 * d * d)
    need = O.mafat_decay_workspace(c)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    O.mafat_decay_attention(c, q.data_ptr(), k.data_ptr(), v.data_ptr(), decay.data_ptr(), None, states.data_ptr(), None,
                            buf.data_ptr() + 6, ws.data_ptr() if need else None, need, M._stream_handle(None))
    torch.cuda.synchronize()
    y = buf[3:3 + rows * row].view(rows, row)
    assert torch.equal(torch.stack([y[:, :d], y[:, head:head + d]], 1), want)
    assert (y[:, d:head] == 7).all() and (y[:, head + d:] == 7).all() and (buf[:3] == 7).all() and (buf[3 + rows * row:] == 7).all()
