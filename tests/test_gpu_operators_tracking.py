"""What autograd is told of the operators, which work through addresses: tensors that they write in place count as changed, and
tangents of forward mode are refused as gradients are."""
import pytest

from gpu_util import require_gpu


def _tokens():
    import torch
    from paper_2107_06960_amd import operators as O
    q, k, v = (torch.randn(4, 2, 32, device="cuda").bfloat16() for _ in range(3))
    return q, k, v, -torch.rand(2, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda"), O.rotary_turns(16)


@pytest.mark.gpu
def test_tensors_written_in_place_count_as_changed():
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    q, k, v, decay, positions, turns = _tokens()
    before = [t._version for t in (q, k)]
    O.rotary(q, positions, turns, k=k)
    assert [t._version for t in (q, k)] == before
    O.rotary(q, positions, turns, k=k, in_place=True)
    assert all(t._version > b for t, b in zip((q, k), before))
    states = torch.zeros(1, 2, 32, 32, device="cuda")
    before = states._version
    O.decay_attention(q, k, v, decay, states=states)
    assert states._version > before
    # views share their base's count, and an outer graph refuses its backward pass instead of giving wrong gradients
    x = torch.randn(4, 4, 32, device="cuda")
    weight = torch.ones(4, 4, 32, device="cuda", requires_grad=True)
    loss = (x * weight).sum()
    with torch.no_grad():
        O.rotary(x[:, :2], positions, turns, k=x[:, 2:], in_place=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.gpu
def test_tensors_of_inference_mode():
    """They have no count of changes."""
    require_gpu()
    import torch
    from paper_2107_06960_amd import operators as O
    with torch.inference_mode():
        q, k, v, decay, positions, turns = _tokens()
        states = torch.zeros(1, 2, 32, 32, device="cuda")
        O.rotary(q, positions, turns, k=k, in_place=True)
        assert torch.isfinite(O.decay_attention(q, k, v, decay, states=states)).all() and states.abs().sum() > 0


@pytest.mark.gpu
def test_tangents_are_refused():
    require_gpu()
    import torch
    import torch.autograd.forward_ad as forward
    from paper_2107_06960_amd import operators as O
    q, k, v, decay, positions, turns = _tokens()
    x, gain = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    w, s = torch.zeros(8, 64, device="cuda").to(O.F8), torch.ones(8, device="cuda")
    x8, x_scale = x.to(O.F8), torch.ones(4, device="cuda")
    a, b = torch.zeros(1, 2, 64, device="cuda").bfloat16(), torch.zeros(1, 8, 2, device="cuda").bfloat16()
    of_row = torch.zeros(4, dtype=torch.int32, device="cuda")
    states, maps = torch.zeros(1, 2, 32, 32, device="cuda"), torch.randn(1, 9, 2, 32, device="cuda").bfloat16()
    calls = [(lambda x, gain, r: O.add_rms_norm(x, gain, r), (x, gain, x.clone())),
             (lambda x_scale, s, bias: O.linear8(x8, x_scale, w, s, bias=bias), (x_scale, s, s.clone())),
             (lambda a, b, f: O.linear8(x8, x_scale, w, s, adapters=(a, b, f), row_adapter=of_row), (a, b, torch.ones(1, device="cuda"))),
             (lambda q, k, v: O.cross_attention(q, k, v), (q, maps, maps.clone())),
             (lambda q, k, t: O.rotary(q, positions, t, k=k), (q, k, turns)),
             (lambda q, k, t: O.rotary(q, positions, t, k=k, in_place=True), (q.clone(), k.clone(), turns)),
             (lambda q, k, v, g, st: O.decay_attention(q, k, v, g, states=st), (q, k, v, decay, states)),
             (lambda x, a, g, s, r, b: O.block_norm(x, after_gain=a, gate=g, scale=s, residual=r, before_gain=b),
              (x, gain, x.clone(), gain.clone(), x.clone(), gain.clone()))]
    for call, tensors in calls:
        call(*tensors)
        with forward.dual_level():
            call(*tensors)  # no tangents, nothing lost
            for i, t in enumerate(tensors):
                with pytest.raises(ValueError, match="forward only"):
                    call(*(forward.make_dual(u, torch.ones_like(u)) if j == i else u for j, u in enumerate(tensors)))
        assert all(not hasattr(t, "grad_fn") or t.grad_fn is None for t in tensors)
