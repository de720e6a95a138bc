"""Single products of the gated delta rule in fp32: keys of one channel and no writes leave o = q S, one product of pairs of
tf32 values.

Both first parts are rounded to 11 bits, so that the second parts are below 2^-11 of 2^e (e the value's exponent) and are cut
off at 2^-22 of it; what is left out is the product of the second parts.  Worst case 2 * 2^-22 + 2^-22 and the
rounding of the sum, 2^-24: 7.8e-7.  The parts left out have either sign: a mean of 2^16 products deviates by
their size, 1.5e-7 at most (rms), over 2^8, 6e-10; five of these and 1e-8 for the uneven density of the values are allowed."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_products_are_not_biased():
    import paper_2412_16602_gb300 as vmb
    gen = torch.Generator().manual_seed(5)
    T, H, Dv = 64, 4, 256
    q, S = 1 + torch.rand(1, T, H, 1, generator=gen), 1 + torch.rand(1, H, 1, Dv, generator=gen)
    S[:, 1] *= -1
    z = torch.zeros(1, T, H, device="cuda")
    o = vmb.vmb_delta_rule_fwd(q.cuda(), torch.zeros_like(q).cuda(), torch.zeros(1, T, H, Dv, device="cuda"), z, z,
                               initial_state=S.cuda(), scale=1.0)[0]
    off = o.double().cpu() / (q.double() * S.double().transpose(1, 2)) - 1  # [1, T, H, Dv]
    assert off.abs().max().item() <= 7.8e-7
    assert abs(off.mean().item()) <= 1.3e-8
