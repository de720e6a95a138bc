"""A channels-last token mixer over maps and videos, built from this library's operators: group norm with an activation,
rotary positions of time, row and column on the queries and keys, and the gated delta rule over the tokens.

    python examples/delta_mixer.py [--steps N]

trains a mixer block to undo noise on small synthetic videos, then streams a video through it: the first frames as one
prefill, the tokens of the next frame one at a time from the state that the prefill left.  Needs a GPU and the built
library.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2412_16602_gb300 as vmb  # noqa: E402


class GroupNormAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, act):
        y, stats = vmb.vmb_group_norm_fwd(x, weight, bias, groups, act=act, want_stats=True)
        ctx.save_for_backward(x, weight, bias, stats)
        ctx.groups, ctx.act = groups, act
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, bias, stats = ctx.saved_tensors
        d = vmb.vmb_group_norm_bwd(x, weight, bias, stats, dy.contiguous(), ctx.groups, act=ctx.act)
        return d["x"], d["weight"], d["bias"], None, None


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, freq, sections, grid):
        ctx.freq, ctx.kw = freq, dict(sections=sections, grid=grid)
        return vmb.vmb_rotary_fwd(q, k, freq, **ctx.kw)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        dq, dk = vmb.vmb_rotary_fwd(dq.contiguous(), dk.contiguous(), ctx.freq, inverse=True, **ctx.kw)
        return dq, dk, None, None, None


class DeltaRule(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        o, _, saved = vmb.vmb_delta_rule_fwd(q, k, v, g, beta, want_saved=True)
        ctx.save_for_backward(q, k, v, g, beta, saved)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        *inputs, saved = ctx.saved_tensors
        d = vmb.vmb_delta_rule_bwd(*inputs, do.contiguous(), saved)
        return d["q"], d["k"], d["v"], d["g"], d["beta"]


class DeltaMixer(torch.nn.Module):
    """x [B, frames, H, W, C] -> the same shape: norm each frame, mix the tokens of all frames in order, add."""

    def __init__(self, channels, key_heads, value_heads, key_dim, groups=4, sections=(4, 6, 6)):
        super().__init__()
        self.Hk, self.Hv, self.Dk, self.Dv = key_heads, value_heads, key_dim, channels // value_heads
        self.groups, self.sections = groups, sections
        self.norm_weight, self.norm_bias = torch.nn.Parameter(torch.ones(channels)), torch.nn.Parameter(torch.zeros(channels))
        self.w_qkv = torch.nn.Linear(channels, 2 * key_heads * key_dim + channels, bias=False)
        self.w_gates = torch.nn.Linear(channels, 2 * value_heads)
        self.w_out = torch.nn.Linear(channels, channels)
        self.register_buffer("freq", torch.cat([100.0 ** (-torch.arange(n) / n) for n in sections]).float())

    def project(self, x):
        """q, k, v, g, beta of the tokens of frames x [B, frames, H, W, C]."""
        B, C = x.shape[0], x.shape[-1]
        y = GroupNormAct.apply(x.reshape(-1, *x.shape[2:]), self.norm_weight, self.norm_bias, self.groups, "silu").reshape(B, -1, C)
        q, k, v = self.w_qkv(y).split([self.Hk * self.Dk, self.Hk * self.Dk, C], -1)
        q, k = (F.normalize(t.unflatten(-1, (self.Hk, self.Dk)), dim=-1) for t in (q, k))
        decay, write = self.w_gates(y).chunk(2, -1)
        return q, k, v.unflatten(-1, (self.Hv, self.Dv)), -0.1 * F.softplus(decay).contiguous(), torch.sigmoid(write).contiguous()

    def forward(self, x):
        q, k, v, g, beta = self.project(x)
        q, k = Rotary.apply(q.contiguous(), k.contiguous(), self.freq, self.sections, tuple(x.shape[1:4]))
        return x + self.w_out(DeltaRule.apply(q, k, v.contiguous(), g, beta).flatten(2)).view(x.shape)

    @torch.no_grad()
    def prefill(self, x):
        """The mixed frames and the state after them."""
        q, k, v, g, beta = self.project(x)
        q, k = vmb.vmb_rotary_fwd(q, k, self.freq, sections=self.sections, grid=tuple(x.shape[1:4]))
        o, state, _ = vmb.vmb_delta_rule_fwd(q, k, v, g, beta, want_state=True)
        return x + self.w_out(o.flatten(2)).view(x.shape), state

    @torch.no_grad()
    def stream(self, frame, time, state):
        """The next frame [B, H, W, C] token by token, `state` updated in place."""
        B, H, W, C = frame.shape
        q, k, v, g, beta = self.project(frame.unsqueeze(1))
        at = torch.stack([torch.full((H * W,), time), torch.arange(H * W) // W, torch.arange(H * W) % W])
        at = at.to(torch.int32).unsqueeze(1).expand(3, B, H * W).contiguous().to(frame.device)
        q, k = vmb.vmb_rotary_fwd(q, k, self.freq, at, sections=self.sections)
        o = [vmb.vmb_delta_rule_step(*(t[:, i:i + 1] for t in (q, k, v)), *(t[:, i:i + 1].contiguous() for t in (g, beta)), state)
             for i in range(H * W)]
        return frame + self.w_out(torch.cat(o, 1).flatten(2)).view(frame.shape)


def videos(batch, frames, size, channels, gen):
    """Smooth patterns that move from frame to frame."""
    place = torch.rand(batch, 1, channels, 2, generator=gen, device="cuda") * 6
    speed = torch.randn(batch, 1, channels, 2, generator=gen, device="cuda") * 0.3
    t = torch.arange(frames, device="cuda").view(1, -1, 1, 1)
    phase = place + speed * t
    grid = torch.arange(size, device="cuda") * 0.5
    rows = torch.sin(grid.view(1, 1, -1, 1, 1) + phase[..., 0].unsqueeze(2).unsqueeze(3))
    cols = torch.cos(grid.view(1, 1, 1, -1, 1) + phase[..., 1].unsqueeze(2).unsqueeze(3))
    return (rows * cols).contiguous()


def main(steps=60, seed=0):
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    net = DeltaMixer(channels=64, key_heads=2, value_heads=4, key_dim=32).cuda()
    opt = torch.optim.Adam(net.parameters(), 1e-2)
    losses = []
    for _ in range(steps):
        clean = videos(8, 4, 9, 64, gen)
        noisy = clean + 0.5 * torch.randn(clean.shape, generator=gen, device="cuda")
        loss = F.mse_loss(net(noisy), clean)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    print(f"loss of the first step {losses[0]:.4f}, of the last {losses[-1]:.4f}")

    x = videos(2, 4, 9, 64, gen)
    with torch.no_grad():
        whole = net(x)
    first, state = net.prefill(x[:, :3].contiguous())
    last = net.stream(x[:, 3].contiguous(), 3, state)
    off = (torch.cat([first, last.unsqueeze(1)], 1) - whole).abs().max().item()
    print(f"prefill and steps against the whole video: largest difference {off:.2e}")
    return losses, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    main(ap.parse_args().steps)
