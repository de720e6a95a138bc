"""Packed sequences with a bound of the longest one that is looser than all tokens together: sizes."""
import pytest

MOST = 2147483647


@pytest.mark.parametrize("bound", [1001, 1 << 20, MOST - 63, MOST - 62, MOST])
@pytest.mark.parametrize("B,Hv", [(2, 2), (64, 2), (100, 12)])
def test_sizes_are_those_of_the_tightest_bound(B, Hv, bound):
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    for grads in (False, True):
        want = vmb.vmb_delta_rule_workspace_bytes(B, 1000, 1000, True, 1, Hv, 64, 64, grads)
        assert want > 0 and vmb.vmb_delta_rule_workspace_bytes(B, bound, 1000, True, 1, Hv, 64, 64, grads) == want
    want = vmb.vmb_delta_rule_saved_bytes(B, 1000, 1000, True, Hv, 64, 64)
    assert want > 0 and vmb.vmb_delta_rule_saved_bytes(B, bound, 1000, True, Hv, 64, 64) == want
    assert vmb.vmb_delta_rule_workspace_bytes(B, -1, 1000, True, 1, Hv, 64, 64) == 0
