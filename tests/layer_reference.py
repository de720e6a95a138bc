"""64-bit definitions of the operators of a layer around the scan over tokens, token after token, for the tests."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # the largest relative error of one rounding


def rel(got, want):
    """Relative error in the 2-norm (0 / 0 is 0)."""
    d = (got.double().cpu() - want.double().cpu()).norm()
    n = want.double().norm().cpu()
    return float(d / n) if n > 0 else float(d)


def spans(x, offsets):
    """(batch row, first token, one past the last) of every sequence."""
    if offsets is None:
        return [(b, 0, x.shape[1]) for b in range(x.shape[0])]
    at = offsets.tolist()
    return [(0, at[i], at[i + 1]) for i in range(len(at) - 1)]


def activation(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z


def conv(x, weight, bias, initial=None, offsets=None, act="silu"):
    """(y, final states) of the short causal convolution."""
    W, rows, last = weight.shape[1], {}, []
    for i, (b, t0, t1) in enumerate(spans(x, offsets)):
        first = x.new_zeros(W - 1, x.shape[2]) if initial is None else initial[i]
        seen = torch.cat([first, x[b, t0:t1]])
        for t in range(t1 - t0):
            z = (seen[t:t + W] * weight.t()).sum(0)
            rows[b, t0 + t] = activation(z if bias is None else z + bias, act)
        last.append(seen[t1 - t0:])
    zero = x.new_zeros(x.shape[2])
    y = [rows.get((b, t), zero) for b in range(x.shape[0]) for t in range(x.shape[1])]
    return torch.stack(y).view(x.shape) if y else x.new_zeros(x.shape), torch.stack(last) if last else x.new_zeros(0, W - 1, x.shape[2])


def scan(x, delta, A, Bm, Cm, skip=None, bias=None, z=None, initial=None, offsets=None, softplus=True):
    """(y, final states) of the selective scan over tokens."""
    D, N = A.shape
    rows, last = {}, []
    raw = delta if bias is None else delta + bias
    dt = torch.logaddexp(raw, torch.zeros((), dtype=raw.dtype, device=raw.device)) if softplus else raw
    for i, (b, t0, t1) in enumerate(spans(x, offsets)):
        h = x.new_zeros(D, N) if initial is None else initial[i]
        for t in range(t0, t1):
            h = torch.exp(dt[b, t].unsqueeze(1) * A) * h + (dt[b, t] * x[b, t]).unsqueeze(1) * Bm[b, t]
            y = h @ Cm[b, t]
            if skip is not None:
                y = y + skip * x[b, t]
            rows[b, t] = y if z is None else y * z[b, t] * torch.sigmoid(z[b, t])
        last.append(h)
    zero = x.new_zeros(D)
    y = [rows.get((b, t), zero) for b in range(x.shape[0]) for t in range(x.shape[1])]
    return torch.stack(y).view(x.shape) if y else x.new_zeros(x.shape), torch.stack(last) if last else x.new_zeros(0, D, N)


def gradients(fn, inputs, outputs_grad):
    """Gradients of sum(fn(*inputs) * outputs_grad) for the 64-bit inputs (None stays None)."""
    leaves = [None if t is None else t.detach().double().cpu().requires_grad_() for t in inputs]
    outs = fn(*leaves)
    live = [t for t in leaves if t is not None]
    total = sum((o * g.double().cpu()).sum() for o, g in zip(outs, outputs_grad) if g is not None)
    got = iter(torch.autograd.grad(total + sum(0.0 * t.sum() for t in live), live))
    return [None if t is None else next(got) for t in leaves]
