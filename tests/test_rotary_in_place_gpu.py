"""Rotary positions in place where a tensor is dense although a stride of its has no meaning (one row, one token)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 12])
@pytest.mark.parametrize("B", [1, 2])
def test_dense_beside_a_strided_one(B, T):
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(2)
    row = torch.randn(B, T, 200, device="cuda")
    q, k = torch.randn(B, T, 2, 32, device="cuda"), row[..., 64:128].unflatten(-1, (2, 32))
    freq = torch.rand(16, device="cuda")
    kw = dict(sections=(16,), grid=(T,))
    a, b = vmb.vmb_rotary_fwd(q, k, freq, **kw)
    c, d = vmb.vmb_rotary_fwd(q, k, freq, q_out=q, **kw)
    assert c is q and torch.equal(q, a) and torch.equal(d, b)
    # the other way round, and a strided tensor in place of itself
    x, y = vmb.vmb_rotary_fwd(k, a, freq, k_out=a, **kw)
    assert y is a and torch.equal(x, b)
    if B * T > 1:
        dense = torch.as_strided(row, (B, T, 2, 32), (T * 64, 64, 32, 1))  # (the same address, other rows)
        with pytest.raises(vmb.VmbError):
            vmb.vmb_rotary_fwd(row[..., :64].unflatten(-1, (2, 32)), None, freq, q_out=dense, **kw)
