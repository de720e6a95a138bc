"""Offsets that decrease or leave the tokens are reported by the scan over tokens and by its gradients, wherever they are, and good ones are not."""
import pytest
import torch

pytestmark = pytest.mark.gpu
GOOD = [[0, 150], [3, 3, 70, 70, 140], [150], [0] * 300 + [150] * 300]
BAD = [[0, 100, 50, 150], [0, 150, 149, 150], [70, 0, 150], [0, 151], [-1, 150], [0, 40, 80, 120, 119], [-1], [151], [0] * 300 + [10, 9] + [150] * 300,
       [0, 1 << 30], [0, -(1 << 31), 150]]


@pytest.mark.parametrize("D", [24, 200])
@pytest.mark.parametrize("at,bad", [(o, False) for o in GOOD] + [(o, True) for o in BAD])
def test_offsets(at, bad, D):
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    T, N = 150, 16
    ins = [r(1, T, D), r(1, T, D), -torch.rand(D, N, device="cuda"), r(1, T, N), r(1, T, N), r(D), r(D) - 2, r(1, T, D)]
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    need = max(vmb.vmb_token_scan_workspace_bytes(len(at) - 1, T, T, True, D, N, grads) for grads in (False, True))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    want = vmb.VMB_ERR_BOUNDS if bad else vmb.VMB_OK
    y, last, saved = vmb.vmb_token_scan_fwd(*ins, offsets=offsets, want_state=True, want_saved=True, workspace=ws)
    assert vmb.vmb_read_status(ws) == want
    saved.zero_()  # (bad offsets may leave some of it as the memory was)
    vmb.vmb_token_scan_bwd(*ins, ins[0], saved, offsets=offsets, workspace=ws)
    assert vmb.vmb_read_status(ws) == want
