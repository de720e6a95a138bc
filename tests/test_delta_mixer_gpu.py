"""The token mixer example: its operators together, in training and in serving."""
import pytest

pytestmark = pytest.mark.gpu


def test_trains_and_streams():
    from examples import delta_mixer
    losses, off = delta_mixer.main(steps=60)
    assert losses[-1] < 0.7 * losses[0]
    # the same sums in another order: fp32 products of up to 64 terms through four layers of them, values below 10
    assert off < 1e-4


def test_gradients_of_the_block_against_differences():
    import torch

    from examples import delta_mixer
    torch.manual_seed(1)
    net = delta_mixer.DeltaMixer(64, 2, 4, 32).cuda()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = delta_mixer.videos(1, 2, 7, 64, gen)
    w = torch.randn(x.shape, generator=gen, device="cuda")
    (net(x) * w).sum().backward()
    for p in net.parameters():
        step = torch.randn(p.shape, generator=gen, device="cuda") * p.detach().abs().mean()
        f = []
        with torch.no_grad():
            for s in (1e-2, -1e-2):
                p += s * step
                f.append((net(x).double() * w.double()).sum().item())
                p -= s * step
        want, size = (p.grad.double() * step.double()).sum().item(), p.grad.norm().item() * step.norm().item() / p.numel() ** 0.5
        # rounding of f (a sum of 6000 terms of fp32 accuracy) over the step, and the second-order term of the step
        assert abs((f[0] - f[1]) / 2e-2 - want) <= 1e-2 * (abs(want) + size) + 2e-3
