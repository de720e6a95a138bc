"""vmb_read_status without a workspace: the errors of every default workspace of the calling thread, whichever operators and streams
they are of, and a captured call's in the workspace that it was given."""
import pytest
import torch

pytestmark = pytest.mark.gpu
T, D, N = 100, 24, 16


@pytest.fixture
def vmb():
    import paper_2412_16602_gb300 as vmb
    vmb.vmb_read_status()  # (whatever earlier calls of this thread have left)
    return vmb


def scan(vmb, last, **kw):
    r = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    offsets = torch.tensor([0, 40, last], dtype=torch.int32, device="cuda")
    return vmb.vmb_token_scan_fwd(r(1, T, D), r(1, T, D), -torch.rand(D, N, device="cuda"), r(1, T, N), r(1, T, N), offsets=offsets, **kw)


@pytest.mark.parametrize("own_stream", [False, True])
def test_of_the_scan_over_tokens(vmb, own_stream):
    stream = torch.cuda.Stream() if own_stream else None
    torch.cuda.synchronize()
    scan(vmb, T, stream=stream)
    assert vmb.vmb_read_status() == vmb.VMB_OK
    scan(vmb, T + 1, stream=stream)
    assert vmb.vmb_read_status() == vmb.VMB_ERR_BOUNDS
    assert vmb.vmb_read_status() == vmb.VMB_OK  # cleared


def test_of_the_delta_rule(vmb):
    from tests import delta_reference as ref
    d = [t.cuda() for t in ref.inputs(1, T, 1, 1, 64, 64, 5)]
    vmb.vmb_delta_rule_fwd(*d, offsets=torch.tensor([0, 40, T + 1], dtype=torch.int32, device="cuda"), max_len=T)
    assert vmb.vmb_read_status() == vmb.VMB_ERR_BOUNDS and vmb.vmb_read_status() == vmb.VMB_OK


def test_of_a_captured_call(vmb):
    n = vmb.vmb_token_scan_workspace_bytes(2, T, T, True, D, N)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    scan(vmb, T, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    offsets = torch.tensor([0, 40, T], dtype=torch.int32, device="cuda")
    x, A, B = torch.randn(1, T, D, device="cuda"), -torch.rand(D, N, device="cuda"), torch.randn(1, T, N, device="cuda")
    with torch.cuda.graph(graph):
        vmb.vmb_token_scan_fwd(x, x, A, B, B, offsets=offsets, workspace=ws)
    for last, want in ((T, vmb.VMB_OK), (T + 7, vmb.VMB_ERR_BOUNDS), (T, vmb.VMB_OK)):
        offsets[2] = last
        graph.replay()
        assert vmb.vmb_read_status(ws) == want


@pytest.mark.parametrize("own_stream", [False, True])
def test_of_a_workspace_that_was_outgrown(vmb, own_stream, monkeypatch):
    """Two small calls that go wrong, each with a larger one after it, before anybody asks."""
    monkeypatch.setattr(vmb.vmb, "_layer_ws", vmb.vmb.Workspace(header=256))
    stream = torch.cuda.Stream() if own_stream else None
    torch.cuda.synchronize()
    for last, n in ((T + 1, 3000), (T, 30000), (T + 1, 100000)):
        scan(vmb, last, stream=stream)
        x, A, B = torch.zeros(1, n, D, device="cuda"), -torch.rand(D, N, device="cuda"), torch.zeros(1, n, N, device="cuda")
        torch.cuda.synchronize()
        before = vmb.layer_workspace(stream=stream).numel()
        vmb.vmb_token_scan_fwd(x, x, A, B, B, stream=stream)
        torch.cuda.synchronize()
        assert vmb.layer_workspace(stream=stream).numel() > before
    assert vmb.vmb_read_status() == vmb.VMB_ERR_BOUNDS
    assert vmb.vmb_read_status() == vmb.VMB_OK  # cleared
