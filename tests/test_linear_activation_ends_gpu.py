"""SiLU and GELU of a product's outputs down to where they leave the type: one rounding to bf16 (2^-8) and 2^-12 for the function, and zero for what lies below
2^-119 (SiLU at -87.3 is 87.3 times the smallest normal fp32 value, the last that the reciprocal keeps)."""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,lo,hi", [("silu", -110.0, -60.0), ("gelu", -20.0, -9.0), ("silu", -0.01, 0.01), ("gelu", -0.01, 0.01)])
@pytest.mark.parametrize("M", [1, 40, 200])
def test_ends(act, lo, hi, M):
    import paper_2412_16602_gb300 as vmb
    z = torch.linspace(lo, hi, 4096, device="cuda")
    x, w = torch.zeros(M, 8, device="cuda", dtype=torch.bfloat16), torch.zeros(4096, 8, device="cuda", dtype=torch.bfloat16)
    y = vmb.vmb_linear_fwd(x, w, z, act=act)[0].double()
    want = ref.activation(z.double(), act).expand(M, -1)
    assert ((y - want).abs() <= (2.0 ** -8 + 2.0 ** -12) * want.abs() + 2.0 ** -119).all()
