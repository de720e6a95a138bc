"""A layer around a selective scan over tokens, built from this library's operators in bf16: root-mean-square norm, a
projection into two halves, the short causal convolution of one half, the selection's projections, the scan with the other half as
its gate, and the projection back to the residual stream.

    python examples/scan_layer.py [--steps N]

trains a layer to continue noisy waves, then serves ragged prompts through it: one packed prefill without padding, then token
after token from the states that it left.  Needs a GPU and the built library.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2412_16602_gb300 as vmb  # noqa: E402


class RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        y, _, _, rstd = vmb.vmb_rms_norm_fwd(x, weight, want_stats=True)
        ctx.save_for_backward(x, weight, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, rstd = ctx.saved_tensors
        d = vmb.vmb_rms_norm_bwd(x, weight, rstd, dy.contiguous())
        return d["x"], d["weight"]


class Linear(torch.autograd.Function):
    """act(x w^T) + residual; the weights are kept in fp32 and used in bf16."""

    @staticmethod
    def forward(ctx, x, weight, act, residual):
        w = weight.to(torch.bfloat16)
        y, pre = vmb.vmb_linear_fwd(x, w, act=act, residual=residual, want_pre=act != "none")
        ctx.save_for_backward(x, w, pre)
        ctx.act, ctx.added = act, residual is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, pre = ctx.saved_tensors
        dy = dy.contiguous()
        d = vmb.vmb_linear_bwd(x, w, dy, pre, act=ctx.act)
        return d["x"], d["weight"].float(), None, dy if ctx.added else None


class CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        ctx.save_for_backward(x, weight, bias)
        return vmb.vmb_causal_conv_fwd(x, weight, bias)[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        d = vmb.vmb_causal_conv_bwd(*ctx.saved_tensors, dy.contiguous())
        return d["x"], d["weight"], d["bias"]


class TokenScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, *inputs):
        y, _, saved = vmb.vmb_token_scan_fwd(*inputs, want_saved=True)
        ctx.save_for_backward(*inputs, saved)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        *inputs, saved = ctx.saved_tensors
        d = vmb.vmb_token_scan_bwd(*inputs, dy.contiguous(), saved)
        return tuple(d[n] for n in ("x", "delta", "A", "B", "C", "Dskip", "delta_bias", "z"))


class ScanLayer(torch.nn.Module):
    """x [B, T, channels] in bf16 -> the same shape."""

    def __init__(self, channels, inner, states=16, rank=16, taps=4):
        super().__init__()
        self.inner, self.states, self.rank, self.taps = inner, states, rank, taps

        def matrix(n, k):
            return torch.nn.Parameter(torch.randn(n, k) / k ** 0.5)

        self.norm = torch.nn.Parameter(torch.ones(channels))
        self.w_in, self.w_sel, self.w_dt, self.w_out = (matrix(2 * inner, channels), matrix(rank + 2 * states, inner),
                                                        matrix(inner, rank), matrix(channels, inner))
        self.filter, self.filter_bias = torch.nn.Parameter(torch.randn(inner, taps) / taps), torch.nn.Parameter(torch.zeros(inner))
        self.A_log = torch.nn.Parameter(torch.arange(1, states + 1).float().log().repeat(inner, 1))
        self.skip = torch.nn.Parameter(torch.ones(inner))
        step = torch.exp(torch.linspace(-6.9, -2.3, inner))  # step sizes 0.001 .. 0.1 where the selection gives nothing
        self.dt_bias = torch.nn.Parameter(step + torch.log(-torch.expm1(-step)))

    def selection(self, u, linear):
        r, Bm, Cm = linear(u, self.w_sel).split([self.rank, self.states, self.states], -1)
        return linear(r, self.w_dt), Bm, Cm

    def forward(self, x):
        def linear(t, w, residual=None):
            return Linear.apply(t, w, "none", residual)

        u, z = linear(RmsNorm.apply(x, self.norm), self.w_in).split(self.inner, -1)
        u = CausalConv.apply(u, self.filter, self.filter_bias)
        delta, Bm, Cm = self.selection(u, linear)
        y = TokenScan.apply(u, delta, -torch.exp(self.A_log), Bm, Cm, self.skip, self.dt_bias, z)
        return linear(y, self.w_out, x)

    def states_for(self, streams):
        return (torch.zeros(streams, self.taps - 1, self.inner, dtype=torch.bfloat16, device=self.norm.device),
                torch.zeros(streams, self.inner, self.states, device=self.norm.device))

    @torch.no_grad()
    def serve(self, x, offsets=None, state=None):
        """x [1, tokens, channels] packed by `offsets` (a prefill from nothing): the outputs and the states after each
        sequence; or x [B, T, channels], the next tokens of every stream whose `state` is given, which moves on in place."""
        def linear(t, w, residual=None):
            return vmb.vmb_linear_fwd(t, w.to(torch.bfloat16), residual=residual)[0]

        u, z = linear(vmb.vmb_rms_norm_fwd(x, self.norm)[0], self.w_in).split(self.inner, -1)
        A = -torch.exp(self.A_log)
        if state is None:
            u, inputs = vmb.vmb_causal_conv_fwd(u, self.filter, self.filter_bias, offsets=offsets, want_state=True)
            y, h, _ = vmb.vmb_token_scan_fwd(u, *self._scan_inputs(u, A, linear), z, offsets=offsets, want_state=True)
            state = (inputs, h)
        else:
            u = vmb.vmb_causal_conv_step(u, self.filter, self.filter_bias, state[0])
            y = vmb.vmb_token_scan_step(u, *self._scan_inputs(u, A, linear), z, state[1])
        return linear(y, self.w_out, x), state

    def _scan_inputs(self, u, A, linear):
        delta, Bm, Cm = self.selection(u, linear)
        return delta, A, Bm, Cm, self.skip, self.dt_bias


def waves(batch, tokens, channels, gen):
    at = torch.arange(tokens, device="cuda").view(1, -1, 1)
    speed, phase = (torch.rand(batch, 1, channels, generator=gen, device="cuda") for _ in range(2))
    return torch.sin(at * (0.05 + 0.3 * speed) + 6.3 * phase)


def main(steps=40, seed=0):
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    net = ScanLayer(64, 128).cuda()
    opt = torch.optim.Adam(net.parameters(), 3e-3)
    losses = []
    for _ in range(steps):
        clean = waves(8, 200, 64, gen)
        noisy = (clean + 0.3 * torch.randn(clean.shape, generator=gen, device="cuda")).to(torch.bfloat16)
        loss = F.mse_loss(net(noisy)[:, :-1].float(), clean[:, 1:])
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    print(f"loss of the first step {losses[0]:.4f}, of the last {losses[-1]:.4f}")

    lengths, more = [37, 1, 90, 64], 3
    x = [waves(1, n + more, 64, gen).to(torch.bfloat16) for n in lengths]
    with torch.no_grad():
        whole = [net(t) for t in x]
    offsets = torch.tensor([0, *torch.tensor(lengths).cumsum(0)], dtype=torch.int32, device="cuda")
    y, state = net.serve(torch.cat([t[:, :n] for t, n in zip(x, lengths)], 1), offsets)
    off = [(a - w[:, :n]).float().abs().max() for a, w, n in zip(y.split(lengths, 1), whole, lengths)]
    for i in range(more):
        y, state = net.serve(torch.cat([t[:, n + i:n + i + 1] for t, n in zip(x, lengths)]), state=state)
        off += [(y[b:b + 1] - w[:, n + i:n + i + 1]).float().abs().max() for b, (w, n) in enumerate(zip(whole, lengths))]
    off = torch.stack(off).max().item()
    print(f"packed prompts and steps against whole sequences: largest difference {off:.2e}")
    return losses, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    main(ap.parse_args().steps)
