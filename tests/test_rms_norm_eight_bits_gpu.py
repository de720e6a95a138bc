"""The norm's 8-bit values are the quotients by their row's scale, rounded once: every bit of them, from the definition's own steps in fp32 (the
statistics and the scale are the call's)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,C,dtype,seed", [(16384, 1536, torch.float32, 0), (16384, 1536, torch.float32, 1), (6000, 4096, torch.bfloat16, 2), (3, 77, torch.float32, 3)])
def test_quotients(rows, C, dtype, seed):
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, C, device="cuda", generator=g).to(dtype)
    y, _, scale, rstd = vmb.vmb_rms_norm_fwd(x, bits8=True, want_stats=True)
    s = x.float() * rstd.unsqueeze(1)
    # quotients in 64 bits, rounded to fp32, are the correctly rounded ones (53 bits are more than twice 24 and two)
    assert torch.equal(scale, (s.abs().amax(1).double() / 448).float())
    want = (s.double() / scale.double().unsqueeze(1)).float().clamp(-448, 448).to(torch.float8_e4m3fn)
    assert torch.equal(y.float(), want.float())


def test_a_row_with_an_infinity_keeps_zeros_beside_it():
    """scale is infinite there: finite values over it are zero, the infinity itself is not a number."""
    import paper_2412_16602_gb300 as vmb
    x = torch.zeros(2, 64, device="cuda")
    x[0], x[1] = 1.0, 2.0
    w = torch.ones(64, device="cuda")
    w[5] = float("inf")
    y, _, scale, _ = vmb.vmb_rms_norm_fwd(x, w, bits8=True)
    v = y.float()
    assert scale.isinf().all() and v[:, 5].isnan().all() and not v[:, :5].any() and not v[:, 6:].any()
