"""A wait of the matrix product that runs out: every warp of the epilogue leaves as a whole, the call's status says so, and the next call
finds everything free again.  The sums of each CTA's first tile are kept back; what waits for them gives up after 4 s."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture
def drop():
    import paper_2412_16602_gb300 as vmb
    vmb.lib.vmb_testing_drop_sums.argtypes = [ctypes.c_int]
    try:
        yield vmb.lib.vmb_testing_drop_sums
    finally:
        vmb.lib.vmb_testing_drop_sums(0)


@pytest.mark.parametrize("M,K,N", [(100, 192, 136), (2500, 200, 2600)])  # one CTA; pairs of CTAs, more than one tile for some
def test_sums_that_never_come(drop, M, K, N):
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = (torch.randn(n, K, device="cuda", generator=g).to(torch.bfloat16) for n in (M, N))
    want = vmb.vmb_linear_fwd(x, w)[0]
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK
    drop(1)
    vmb.vmb_linear_fwd(x, w)
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_ERR_TIMEOUT
    drop(0)
    for _ in range(3):
        assert torch.equal(vmb.vmb_linear_fwd(x, w)[0], want)
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK
