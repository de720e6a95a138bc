"""Packed sequences with a loose bound of the longest one: the bits of the call with the tightest."""
import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bound", [10000, 2147483647])
def test_loose_bound(bound):
    import paper_2412_16602_gb300 as vmb
    lens, (Hk, Hv, D) = (300, 0, 450, 1), (1, 2, 64)
    total = sum(lens)
    q, k, v, g, beta = (t.cuda() for t in ref.inputs(1, total, Hk, Hv, D, D, 61))
    do = torch.randn(1, total, Hv, D, device="cuda")
    offsets = torch.tensor([0, 300, 300, 750, 751], dtype=torch.int32, device="cuda")
    kw = dict(offsets=offsets, max_len=max(lens))
    o, S, saved = vmb.vmb_delta_rule_fwd(q, k, v, g, beta, want_state=True, want_saved=True, **kw)
    d = vmb.vmb_delta_rule_bwd(q, k, v, g, beta, do, saved, want_initial=True, **kw)
    # the C entry points themselves: the Python calls tighten the bound
    N, s = len(lens), torch.cuda.current_stream().cuda_stream
    new = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    ws = torch.zeros(vmb.vmb_delta_rule_workspace_bytes(N, bound, total, True, Hk, Hv, D, D, True), dtype=torch.uint8, device="cuda")
    sv = torch.empty(vmb.vmb_delta_rule_saved_bytes(N, bound, total, True, Hv, D, D), dtype=torch.uint8, device="cuda")
    o2, S2, d2 = new(o), new(S), {n: new(t) for n, t in d.items()}
    p = lambda *ts: [t.data_ptr() for t in ts]  # noqa: E731
    sizes = (N, bound, total, Hk, Hv, D, D, D ** -0.5, 0, ws.data_ptr(), ws.numel(), s)
    assert vmb.lib.vmb_delta_rule_fwd(*p(q, k, v, g, beta), None, None, offsets.data_ptr(), *p(o2, S2, sv), *sizes) == vmb.VMB_OK
    assert vmb.lib.vmb_delta_rule_bwd(*p(q, k, g, beta), None, offsets.data_ptr(), do.data_ptr(), None, *p(sv, *d2.values()), *sizes) == vmb.VMB_OK
    assert vmb.vmb_read_status(ws) == vmb.VMB_OK
    # (the tightest bound is the longest sequence, this one all tokens: chains may be cut elsewhere, sums rounded otherwise)
    close = lambda a, b: (a - b).norm().item() <= 2e-5 * b.norm().item()  # noqa: E731
    assert close(o2, o) and close(S2, S) and all(close(d2[n], d[n]) for n in d)
    # with all tokens as the bound: the same bits
    kw["max_len"] = total
    o, S, saved = vmb.vmb_delta_rule_fwd(q, k, v, g, beta, want_state=True, want_saved=True, **kw)
    d = vmb.vmb_delta_rule_bwd(q, k, v, g, beta, do, saved, want_initial=True, **kw)
    assert torch.equal(o2, o) and torch.equal(S2, S) and all(torch.equal(d2[n], d[n]) for n in d)
