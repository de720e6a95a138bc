"""Workspaces that the device cannot use are refused before anything is launched."""
import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu


def test_workspaces_of_the_host_or_with_gaps():
    import paper_2412_16602_gb300 as vmb
    x = [t.cuda() for t in ref.inputs(1, 8, 1, 1, 16, 16, 3)]
    y = torch.randn(2, 5, 12, device="cuda")
    o, _, saved = vmb.vmb_delta_rule_fwd(*x, want_saved=True)
    stats = vmb.vmb_group_norm_fwd(y, None, None, 3, want_stats=True)[1]
    n = 1 << 22
    for ws in (torch.zeros(n, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(n),
               torch.zeros(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        for call in (lambda: vmb.vmb_delta_rule_fwd(*x, workspace=ws), lambda: vmb.vmb_delta_rule_bwd(*x, o, saved, workspace=ws),
                     lambda: vmb.vmb_group_norm_fwd(y, None, None, 3, workspace=ws),
                     lambda: vmb.vmb_group_norm_bwd(y, None, None, stats, y, 3, workspace=ws)):
            with pytest.raises(ValueError):
                call()
