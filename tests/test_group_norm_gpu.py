"""Group norm with an activation, channels last, against 64 bits.  fp32: a value passes about ten roundings and an
exponential good to 2^-22: 2e-6 of the output's size (2-norm) expected at the worst, 5e-6 allowed, the channel sums
(many terms) 1e-5.  bf16 outputs: their own rounding, 4e-3 allowed."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z


def reference(x, w, b, G, eps, act, dy=None):
    """y and, with dy, the gradients by automatic differentiation of the formula in 64 bits."""
    x, w, b = (t.double().detach().requires_grad_(dy is not None) for t in (x, w, b))
    B, C = x.shape[0], x.shape[-1]
    v = x.reshape(B, -1, G, C // G)
    mean = v.mean((1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean((1, 3), keepdim=True)
    z = ((v - mean) / torch.sqrt(var + eps)).reshape(x.shape) * w + b
    y = act64(z, act)
    if dy is None:
        return y
    return (y.detach(), *torch.autograd.grad(y, (x, w, b), dy.double()))


def rel(a, b):
    return ((a.double().cpu() - b).norm() / b.norm().clamp(min=1e-300)).item()


CASES = [  # B, spatial, C, G
    (1, (1,), 8, 2), (2, (7, 5), 6, 3), (1, (14, 14), 192, 8), (3, (5, 3), 257, 1), (2, (33,), 40, 40), (1, (2, 3, 4), 1536, 6),
    (65, (9,), 32, 4), (2, (300, 17), 96, 32), (1, (4,), 16384, 16), (2, (11, 13), 1030, 5), (4, (64, 64), 64, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_gradients(case, act, dtype):
    import paper_2412_16602_gb300 as vmb
    B, spatial, C, G = case
    dt = TYPES[dtype]
    gen = torch.Generator().manual_seed(C + B)
    x = (torch.randn(B, *spatial, C, generator=gen) * (0.3 + torch.rand(C, generator=gen)) + torch.randn(C, generator=gen)).to(dt)
    w, b, dy = 0.5 + torch.rand(C, generator=gen), torch.randn(C, generator=gen), torch.randn(x.shape, generator=gen).to(dt)
    y, dx, dw, db = reference(x, w, b, G, 1e-5, act, dy)
    gy, stats = vmb.vmb_group_norm_fwd(x.cuda(), w.cuda(), b.cuda(), G, act=act, want_stats=True)
    d = vmb.vmb_group_norm_bwd(x.cuda(), w.cuda(), b.cuda(), stats, dy.cuda(), G, act=act)
    small = 5e-6 if dt == torch.float32 else 4e-3
    assert rel(gy, y) <= small
    v = x.double().reshape(B, -1, G, C // G)
    assert rel(stats[..., 0], v.mean((1, 3))) <= 1e-5
    assert rel(stats[..., 1], 1 / torch.sqrt(v.var((1, 3), correction=0) + 1e-5)) <= 1e-5
    if C // G * math.prod(spatial) > 4:  # (in smaller groups dx is a difference of nearly equal numbers)
        assert rel(d["x"], dx) <= 4 * small
    assert rel(d["weight"], dw) <= 1e-5 and rel(d["bias"], db) <= 1e-5
    bare = vmb.vmb_group_norm_fwd(x.cuda(), None, None, G, act=act)[0]
    assert rel(bare, reference(x, torch.ones(C), torch.zeros(C), G, 1e-5, act)) <= small


def test_mean_far_from_zero():
    """A mean 4000 times the deviation: the variance keeps its digits (x itself carries 2^-24 of the mean)."""
    import paper_2412_16602_gb300 as vmb
    gen = torch.Generator().manual_seed(3)
    x = 4000 + torch.randn(2, 50, 40, 64, generator=gen)
    w, b = torch.ones(64), torch.zeros(64)
    y = reference(x, w, b, 4, 1e-5, "none")
    got, stats = vmb.vmb_group_norm_fwd(x.cuda(), w.cuda(), b.cuda(), 4, want_stats=True)
    v = x.double().reshape(2, -1, 4, 16)
    assert rel(stats[..., 1], 1 / torch.sqrt(v.var((1, 3), correction=0) + 1e-5)) <= 1e-6
    assert rel(got, y) <= 4000 * 2 ** -23  # the stored mean's rounding over the deviation


def test_constant_group_and_large_values():
    import paper_2412_16602_gb300 as vmb
    x = torch.full((2, 6, 8), 3.0)
    x[..., 4:] = torch.randn(2, 6, 4, generator=torch.Generator().manual_seed(4)) * 1e15
    for act in ("none", "silu", "gelu"):
        w, b = torch.ones(8), torch.linspace(-200, 200, 8)
        got, stats = vmb.vmb_group_norm_fwd(x.cuda(), w.cuda(), b.cuda(), 2, act=act, want_stats=True)
        assert rel(got, reference(x, w, b, 2, 1e-5, act)) <= 5e-6
        d = vmb.vmb_group_norm_bwd(x.cuda(), w.cuda(), b.cuda(), stats, torch.ones_like(x).cuda(), 2, act=act)
        assert all(torch.isfinite(t).all() for t in d.values())


def test_what_is_not_finite_stays_in_its_group():
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(6)
    x = torch.randn(2, 40, 32, device="cuda")
    want = vmb.vmb_group_norm_fwd(x, None, None, 4, act="silu")[0]
    x[1, 3, 9] = float("inf")
    got = vmb.vmb_group_norm_fwd(x, None, None, 4, act="silu")[0]
    assert torch.equal(got[0], want[0])
    assert torch.equal(got[1, :, :8], want[1, :, :8]) and torch.equal(got[1, :, 16:], want[1, :, 16:])
    assert not torch.isfinite(got[1, 3, 9])


def test_gradient_against_differences():
    """Slopes of the GPU's forward along random directions (fp32, step 1e-2): 2e-3 allowed."""
    import paper_2412_16602_gb300 as vmb
    gen = torch.Generator().manual_seed(5)
    x, w, b = torch.randn(2, 30, 24, generator=gen), 0.5 + torch.rand(24, generator=gen), torch.randn(24, generator=gen)
    dy = torch.randn(x.shape, generator=gen)
    stats = vmb.vmb_group_norm_fwd(x.cuda(), w.cuda(), b.cuda(), 3, act="gelu", want_stats=True)[1]
    d = vmb.vmb_group_norm_bwd(x.cuda(), w.cuda(), b.cuda(), stats, dy.cuda(), 3, act="gelu")
    for i, n in enumerate(("x", "weight", "bias")):
        step = torch.randn((x, w, b)[i].shape, generator=gen)
        f = []
        for s in (1e-2, -1e-2):
            a = [(t + s * step if j == i else t).cuda() for j, t in enumerate((x, w, b))]
            f.append((vmb.vmb_group_norm_fwd(*a, 3, act="gelu")[0].double().cpu() * dy.double()).sum().item())
        want = (d[n].double().cpu() * step.double()).sum().item()
        assert abs((f[0] - f[1]) / 2e-2 - want) <= 2e-3 * d[n].double().norm().item() * step.double().norm().item() / step.numel() ** 0.5 + 2e-3 * abs(want)


def test_workspace_serves_calls_of_any_size_in_turn():
    """Odd addresses give the same values up to rounding, repeated calls the same bits."""
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(7)
    shapes = [(1, 9, 64), (100, 30, 32), (3, 1000, 48), (70, 5, 16)]
    xs = [torch.randn(s, device="cuda") for s in shapes]
    first = [vmb.vmb_group_norm_fwd(x, None, None, 4)[0] for x in xs]
    for _ in range(3):
        for x, y in zip(xs, first):
            assert torch.equal(vmb.vmb_group_norm_fwd(x, None, None, 4)[0], y)
            stats = vmb.vmb_group_norm_fwd(x, None, None, 4, want_stats=True)[1]
            d = vmb.vmb_group_norm_bwd(x, None, None, stats, x, 4)
            e = vmb.vmb_group_norm_bwd(x, None, None, stats, x, 4)
            assert torch.equal(d["x"], e["x"])
    x = torch.randn(2 * 30 * 32 + 1, device="cuda")[1:].view(2, 30, 32)
    a, b = vmb.vmb_group_norm_fwd(x, None, None, 4)[0], vmb.vmb_group_norm_fwd(x.clone(), None, None, 4)[0]
    assert (a - b).abs().max().item() <= 2e-6


def test_refusals_and_empty():
    import paper_2412_16602_gb300 as vmb
    x, w = torch.randn(2, 5, 12, device="cuda"), torch.ones(12, device="cuda")
    for bad in (lambda: vmb.vmb_group_norm_fwd(x, w, w, 5), lambda: vmb.vmb_group_norm_fwd(x, w[:4], None, 3),
                lambda: vmb.vmb_group_norm_fwd(x, w.bfloat16(), None, 3), lambda: vmb.vmb_group_norm_fwd(x.cpu(), w, w, 3),
                lambda: vmb.vmb_group_norm_fwd(x, w, w, 3, act="relu"), lambda: vmb.vmb_group_norm_fwd(x.transpose(0, 1), w, w, 3),
                lambda: vmb.vmb_group_norm_bwd(x, w, w, None, x, 3), lambda: vmb.vmb_group_norm_bwd(x, w, w, x, x, 3)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        vmb.vmb_group_norm_fwd(x.half(), w, w, 3)
    with pytest.raises(vmb.VmbError) as e:
        vmb.vmb_group_norm_fwd(x, w, w, 3, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == vmb.VMB_ERR_WORKSPACE
    y, stats = vmb.vmb_group_norm_fwd(x[:0], w, w, 3, want_stats=True)
    assert y.shape == (0, 5, 12) and stats.shape == (0, 3, 2)
    d = vmb.vmb_group_norm_bwd(x[:0], w, w, stats, x[:0], 3)
    assert d["weight"].abs().max().item() == 0 and d["bias"].abs().max().item() == 0
