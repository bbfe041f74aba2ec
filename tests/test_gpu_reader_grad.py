"""The reader's operators are forward only: while gradients are recorded, a tensor that requires one is refused."""
import pytest

from gpu_util import require_gpu


def _calls():
    """(operator, its tensors by name, a call of them)"""
    import torch
    from paper_2107_06960_amd import operators as O

    def f(*shape):
        return torch.randn(*shape, device="cuda")

    def f8(*shape):
        return f(*shape).to(O.F8)

    of_row = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    norm = dict(x=f(3, 64), gain=f(64), residual=f(3, 64))
    linear = dict(x_scale=f(3), w_scale=f(32), bias=f(32), a=f(2, 4, 64).bfloat16(), b=f(2, 32, 4).bfloat16(), factor=f(2))
    x, w = f8(3, 64), f8(32, 64)
    cross = dict(q=f(4, 2, 64), k=f(2, 9, 1, 64), v=f(2, 9, 1, 64), scale=torch.tensor(0.1))
    return [("norm", norm, lambda t: O.add_rms_norm(t["x"], t["gain"], t["residual"])[0]),
            ("linear", linear, lambda t: O.linear8(x, t["x_scale"], w, t["w_scale"], t["bias"], (t["a"], t["b"], t["factor"]),
                                                   of_row)),
            ("cross", cross, lambda t: O.cross_attention(**t)[0])]


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2])
def test_tensors_that_require_gradients(which):
    require_gpu()
    import torch
    _, tensors, call = _calls()[which]
    want = call(tensors)
    for name in tensors:
        t = dict(tensors, **{name: tensors[name].clone().requires_grad_()})
        with pytest.raises(ValueError, match="forward only"):
            call(t)
        for quiet in (torch.no_grad, torch.inference_mode):
            with quiet():
                assert torch.equal(call(t), want)
        assert torch.equal(call(dict(t, **{name: t[name].detach()})), want)
