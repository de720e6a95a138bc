"""The operators of a layer together: the example in training and serving, its gradients, streams, captured graphs, and
tensors beyond 2^31 elements."""
import math

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def test_example_runs():
    from examples import scan_layer
    losses, off = scan_layer.main(steps=5)
    assert all(math.isfinite(v) for v in losses)
    # six operators, each rounded to bf16 (2^-8 relative) after sums in another order: values below 8 differ by less than six steps of 2^-8
    assert off <= 6 * 8 * 2.0 ** -8


def layer64(net, x):
    """The layer in 64 bits from the same parameters (weights rounded to bf16 as it uses them)."""
    p = {n: (t.detach().to(BF16) if n.startswith("w_") else t.detach()).double().cpu().requires_grad_() for n, t in net.named_parameters()}
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * p["norm"]
    u, z = (y @ p["w_in"].t()).split(net.inner, -1)
    u, _ = ref.conv(u, p["filter"], p["filter_bias"])
    r, Bm, Cm = (u @ p["w_sel"].t()).split([net.rank, net.states, net.states], -1)
    o, _ = ref.scan(u, r @ p["w_dt"].t(), -torch.exp(p["A_log"]), Bm, Cm, p["skip"], p["dt_bias"], z)
    return o @ p["w_out"].t() + x, p


def test_gradients_of_the_layer():
    """Against automatic differentiation of the definition.  Some sixteen roundings of at most 2^-8, forth and back, lie between a loss and
    a parameter; each changes a gradient's norm by no more than that: 2^-4."""
    from examples import scan_layer
    torch.manual_seed(2)
    net = scan_layer.ScanLayer(48, 72, states=8, rank=8).cuda()
    x = torch.randn(2, 45, 48, device="cuda").to(BF16).requires_grad_()
    w = torch.randn(2, 45, 48, device="cuda")
    y = net(x)
    (y.float() * w).sum().backward()
    x64 = x.detach().double().cpu().requires_grad_()
    y64, p = layer64(net, x64)
    (y64 * w.double().cpu()).sum().backward()
    assert ref.rel(y.detach(), y64.detach()) <= 6 * 2.0 ** -8
    assert ref.rel(x.grad, x64.grad) <= 2.0 ** -4
    for n, t in net.named_parameters():
        assert ref.rel(t.grad, p[n].grad) <= 2.0 ** -4, n


@pytest.fixture
def calls(monkeypatch):
    """(call(stream), its result alone): scans cut into segments, gradients, a product in parts, few and many rows."""
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    ins = [r(1, 900, 72), r(1, 900, 72), -torch.rand(72, 16, device="cuda", generator=g) * 4, r(1, 900, 16), r(1, 900, 16), r(72), r(72) - 2, r(1, 900, 72)]
    x, f, b = r(2, 700, 96).to(BF16), r(96, 4), r(96)
    a, w, dy = r(6000, 64).to(BF16), r(40, 64).to(BF16), r(6000, 40).to(BF16)
    few = r(3, 64).to(BF16)

    def scan(stream=None):
        y, h, saved = vmb.vmb_token_scan_fwd(*ins, want_state=True, want_saved=True, stream=stream)
        return [y, h, *vmb.vmb_token_scan_bwd(*ins, ins[0], saved, stream=stream).values()]

    def conv(stream=None):
        y, h = vmb.vmb_causal_conv_fwd(x, f, b, want_state=True, stream=stream)
        return [y, h, *vmb.vmb_causal_conv_bwd(x, f, b, y, stream=stream).values()]

    def norm(stream=None):
        y, t, _, rstd = vmb.vmb_rms_norm_fwd(x, b, x, want_stats=True, stream=stream)
        return [y, t, rstd, *vmb.vmb_rms_norm_bwd(t, b, rstd, y, dsum=x, stream=stream).values()]

    def linear(stream=None):
        y, pre = vmb.vmb_linear_fwd(a, w, act="gelu", want_pre=True, stream=stream)
        return [y, pre, vmb.vmb_linear_fwd(few, w, stream=stream)[0],
                *vmb.vmb_linear_bwd(a, w, dy, pre, act="gelu", want_bias=True, stream=stream).values()]

    fs = [scan, conv, norm, linear]
    alone = [[t.clone() for t in f()] for f in fs]
    torch.cuda.synchronize()
    monkeypatch.setattr(vmb.vmb, "_layer_ws", vmb.vmb.Workspace(header=256))
    return list(zip(fs, alone))


def same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


def test_streams_side_by_side(calls):
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [(f(s), want) for _ in range(4) for s in streams for f, want in calls]
    torch.cuda.synchronize()
    assert all(same(g, want) for g, want in got)


def test_two_captured_graphs_replayed_at_once(calls):
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = [f() for f, _ in calls]
        graphs.append((g, outs, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for g, outs, s in graphs:
            for o in outs:
                for t in o:
                    t.zero_()
        torch.cuda.synchronize()
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        eager = [f() for f, _ in calls]
        torch.cuda.synchronize()
        for outs in (*(o for _, o, _ in graphs), eager):
            assert all(same(o, want) for o, (_, want) in zip(outs, calls))


def test_beyond_two_to_the_31():
    """Rows at the far end of tensors of more than 2^31 elements, against the same rows in a small tensor."""
    import paper_2412_16602_gb300 as vmb
    C, T = 4096, 530_000
    x = torch.zeros(1, T, C, dtype=BF16, device="cuda")
    assert x.numel() > 2 ** 31
    x[:, -40:] = torch.randn(40, C, device="cuda")
    tail = x[:, -40:].clone()
    w, f = torch.randn(C, device="cuda"), torch.randn(C, 4, device="cuda")
    y = vmb.vmb_rms_norm_fwd(x, w)[0]
    assert torch.equal(y[:, -40:], vmb.vmb_rms_norm_fwd(tail, w)[0])
    y = vmb.vmb_causal_conv_fwd(x, f, y=y)[0]
    assert torch.equal(y[:, -40:], vmb.vmb_causal_conv_fwd(tail, f)[0])
    # (tokens of zeros before the tail leave a state of zeros)
    Bm = torch.zeros(1, T, 2, dtype=BF16, device="cuda")
    Bm[:, -40:] = torch.randn(40, 2, device="cuda")
    A = -torch.rand(C, 2, device="cuda")
    y, last, _ = vmb.vmb_token_scan_fwd(x, x, A, Bm, Bm, y=y, want_state=True)
    small, h, _ = vmb.vmb_token_scan_fwd(tail, tail, A, Bm[:, -40:].contiguous(), Bm[:, -40:].contiguous(), want_state=True)
    assert ref.rel(y[:, -40:], small) <= 2.0 ** -8 and ref.rel(last, h) <= 2.0 ** -15
    m = (torch.randn(8, C, device="cuda") / 64).to(BF16)
    # (a small tensor's contraction may be split, its sums are then in another order: both are within one rounding and the 4096^1.5 2^-24 that the
    # sums of so many terms of random sign can be off by of the product)
    assert ref.rel(vmb.vmb_linear_fwd(x.view(T, C), m)[0][-40:], tail[0].double() @ m.double().t()) <= 2.0 ** -8 + C ** 1.5 * 2.0 ** -24
    del y
    out = vmb.vmb_linear_fwd(x.view(T, C)[:, :64], (torch.randn(C + 8, 64, device="cuda") / 8).to(BF16))[0]
    assert out.numel() > 2 ** 31 and not out[:100].any() and out[-40:].float().norm() > 0
