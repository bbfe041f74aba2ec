"""What autograd is told of the operators, which work through addresses: tensors that they write in place count as
changed."""
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
