"""Rotary positions beyond 2^24, which a float does not hold, at angles of every size."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_angles_at_far_positions():
    """Turned unit pairs are (cos, sin) themselves.  The angle: 2^-24 of a turn; its sine and cosine: two units in the last
    place of one, 2^-23; two roundings more, 2^-24 each."""
    import paper_2412_16602_gb300 as vmb
    places = [(1 << 24) + 1, (1 << 24) + 3, (1 << 25) + 2, (1 << 30) + 33, 2147483647, -(1 << 24) - 1, -2147483647, -2147483648, 1 << 24, 12345]
    freq = torch.tensor([5e-5, 6e-5, 9e-7, 4.7e-7, 3e-8, 1e-9, 1e-4, 0.37, 1.0, 3.0])
    q = torch.zeros(1, len(places), 1, 20)
    q[..., :10] = 1
    at = torch.tensor(places, dtype=torch.int32).view(1, 1, -1)
    got = vmb.vmb_rotary_fwd(q.cuda(), None, freq.cuda(), at.cuda(), sections=(10,))[0].double().cpu()[0, :, 0]
    angle = torch.tensor(places, dtype=torch.float64)[:, None] * freq.double()
    # (the product of a 31-bit place and a 24-bit frequency, rounded to 53 bits, and its reduction: below 1e-6 at 6e9)
    off = torch.maximum((got[:, :10] - torch.cos(angle)).abs(), (got[:, 10:] - torch.sin(angle)).abs())
    limit = 6.2832 * 2 ** -24 + 2 ** -23 + 2 * 2 ** -24 + angle.abs() * 2 ** -53
    assert (off <= limit).all(), (off / limit).max().item()
