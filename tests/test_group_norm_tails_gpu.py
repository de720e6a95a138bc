"""The activations value by value where they are small: with a weight of zero the norm passes the bias on exactly, so that
y = act(bias) and dbias = the number of pixels times act'(bias), whatever x is.

Computed in fp32: an exponential whose argument of up to 17 (SiLU at -12) or 72 (GELU, z^2 / 2) is rounded, 2^-24 of it, and
a few operations, 1e-5 in all.  bf16 values lie between the roundings of both ends of that interval.  The slopes are sums in
fp32 of either type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def value(z, act):
    return z * torch.sigmoid(z) if act == "silu" else 0.5 * z * torch.erfc(-z / math.sqrt(2))


def slope(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def run(act, dtype, C, L):
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(C)
    x = torch.randn(2, L, C, device="cuda").to(TYPES[dtype])
    bias = torch.linspace(-12, -3, C)
    y, stats = vmb.vmb_group_norm_fwd(x, torch.zeros(C, device="cuda"), bias.cuda(), 2, act=act, want_stats=True)
    d = vmb.vmb_group_norm_bwd(x, torch.zeros(C, device="cuda"), bias.cuda(), stats, torch.ones_like(x), 2, act=act)
    z, y = bias.double(), y.cpu()
    if dtype == "f32":
        off = (y.double() / value(z, act) - 1).abs().max().item()
        assert off <= 1e-5, off
    else:  # (the values are negative)
        assert (y >= (value(z, act) * (1 + 1e-5)).bfloat16()).all() and (y <= (value(z, act) * (1 - 1e-5)).bfloat16()).all()
    off = (d["bias"].double().cpu() / (2 * L * slope(z, act)) - 1).abs().max().item()
    assert off <= 1e-5, off


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,L", [(512, 20), (514, 20), (1024, 3000)])  # a cluster, single values, two passes over memory
def test_silu(dtype, C, L):
    run("silu", dtype, C, L)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,L", [(512, 20), (514, 20), (1024, 3000)])
def test_gelu(dtype, C, L):
    run("gelu", dtype, C, L)
