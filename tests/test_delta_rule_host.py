"""The 64-bit reference of the gated delta rule: closed forms, and its gradients against differences."""
import torch

from tests import delta_reference as ref


def test_one_token():
    q, k, v, g, beta = ref.inputs(2, 1, 1, 2, 5, 3, 0)
    o, S, _ = ref.forward(q, k, v, g, beta)
    for h in range(2):
        u = beta[:, 0, h, None].double() * v[:, 0, h].double()
        assert torch.allclose(S[:, h], torch.einsum("bk,bv->bkv", k[:, 0, 0].double(), u))
        qk = (q[:, 0, 0].double() * k[:, 0, 0].double()).sum(-1, keepdim=True)
        assert torch.allclose(o[:, 0, h], 5 ** -0.5 * qk * u)


def test_a_key_written_with_beta_one_is_read_back():
    q, k, v, g, beta = ref.inputs(1, 6, 1, 1, 8, 4, 1)
    o, _, _ = ref.forward(k, k, v, g, torch.ones_like(beta), scale=1.0)
    assert torch.allclose(o, v.double(), atol=1e-6)  # keys are of length one up to fp32 rounding


def test_gradients_against_differences():
    x = [t.double() for t in ref.inputs(2, 7, 1, 2, 4, 3, 2)]
    gen = torch.Generator().manual_seed(3)
    do, dfinal, init = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((2, 7, 2, 3), (2, 2, 4, 3), (2, 2, 4, 3)))
    d = ref.backward(*x, do, init, dfinal)

    def loss(y, s):
        o, S, _ = ref.forward(*y, s)
        return ((o * do).sum() + (S * dfinal).sum()).item()

    for i, name in enumerate(("q", "k", "v", "g", "beta", "initial_state")):
        args = x + [init]
        step = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = ([a + s * 1e-5 * step if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        slope = (loss(up[:5], up[5]) - loss(down[:5], down[5])) / 2e-5
        want = (d[name] * step).sum().item()
        assert abs(slope - want) <= 1e-7 * max(1.0, abs(want)), name
