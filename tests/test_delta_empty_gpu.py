"""Heads or channels of none: outputs and gradients that have elements are sums of nothing, zero."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(1, 2, 0, 8), (1, 2, 8, 0), (2, 0, 8, 8)])
def test_sums_of_nothing(Hk, Hv, Dk, Dv):
    import paper_2412_16602_gb300 as vmb
    new = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    rubbish = [torch.full((n,), float("nan"), device="cuda") for n in (24, 48, 96, 192) * 8]
    del rubbish
    x = [new(2, 3, Hk, Dk), new(2, 3, Hk, Dk), new(2, 3, Hv, Dv), -new(2, 3, Hv), new(2, 3, Hv)]
    o, S, saved = vmb.vmb_delta_rule_fwd(*x, want_state=True, want_saved=True)
    d = vmb.vmb_delta_rule_bwd(*x, x[2], saved)
    step = vmb.vmb_delta_rule_step(*x, new(2, Hv, Dk, Dv))
    assert S.shape == (2, Hv, Dk, Dv)
    for t, want in [(o, x[2]), (step, x[2]), *zip((d[n] for n in ("q", "k", "v", "g", "beta")), x)]:
        assert t.shape == want.shape and (t == 0).all()
