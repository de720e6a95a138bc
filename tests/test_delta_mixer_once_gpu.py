"""The token mixer example's autograd functions have first derivatives only: a second one is refused, not lost."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_second_derivatives_are_refused():
    from examples import delta_mixer as m
    torch.manual_seed(4)
    new = lambda *s: torch.randn(s, device="cuda", requires_grad=True)  # noqa: E731
    x, w, b = new(2, 6, 8), new(8), new(8)
    q, k, v, g, beta = new(1, 6, 1, 8), new(1, 6, 1, 8), new(1, 6, 1, 8), new(1, 6, 1), new(1, 6, 1)
    for out, of in ((m.GroupNormAct.apply(x, w, b, 2, "silu"), x), (m.DeltaRule.apply(q, k, v, g, beta), q),
                    (m.Rotary.apply(q, k, torch.rand(4, device="cuda"), (4,), (6,))[0], q)):
        d, = torch.autograd.grad(out.square().sum(), of, create_graph=True)
        assert torch.isfinite(d).all()
        with pytest.raises(RuntimeError):
            (d.square().sum() + of.square().sum()).backward()  # a gradient penalty beside another term
