"""The gated delta rule, token by token in 64 bits on the CPU, and its gradients by the reverse recurrence
(written from the recurrence's derivative; test_delta_rule_host.py checks them against differences)."""
import torch


def unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def inputs(B, T, Hk, Hv, Dk, Dv, seed, dtype=torch.float32, g_scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    q, k = unit(n(B, T, Hk, Dk) + 0.5 * n(1, 1, Hk, Dk)), unit(n(B, T, Hk, Dk) + 0.5 * n(1, 1, Hk, Dk))
    g = -g_scale * torch.exp(2 * n(B, T, Hv) - 3)
    return [x.to(dtype) for x in (q, k, n(B, T, Hv, Dv), g, torch.sigmoid(n(B, T, Hv)))]


def forward(q, k, v, g, beta, initial=None, scale=None):
    """o, final state, and what the gradients need; [B, T, H, D] in float64."""
    B, T, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    scale = Dk ** -0.5 if scale is None else scale
    q, k, v, g, beta = (x.double() for x in (q, k, v, g, beta))
    qr, kr = q.repeat_interleave(Hv // Hk, 2), k.repeat_interleave(Hv // Hk, 2)
    S = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64) if initial is None else initial.double()
    o, kept = torch.zeros(B, T, Hv, Dv, dtype=torch.float64), []
    for t in range(T):
        decayed = S * torch.exp(g[:, t])[..., None, None]
        r = v[:, t] - torch.einsum("bhkv,bhk->bhv", decayed, kr[:, t])
        S = decayed + torch.einsum("bhk,bhv->bhkv", kr[:, t], beta[:, t, :, None] * r)
        o[:, t] = scale * torch.einsum("bhkv,bhk->bhv", S, qr[:, t])
        kept.append((decayed, r, S))
    return o, S, kept


def backward(q, k, v, g, beta, do, initial=None, dfinal=None, scale=None):
    B, T, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    scale = Dk ** -0.5 if scale is None else scale
    kept = forward(q, k, v, g, beta, initial, scale)[2]
    q, k, v, g, beta, do = (x.double() for x in (q, k, v, g, beta, do))
    qr, kr = q.repeat_interleave(Hv // Hk, 2), k.repeat_interleave(Hv // Hk, 2)
    dS = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64) if dfinal is None else dfinal.double()
    d = dict(q=torch.zeros_like(qr), k=torch.zeros_like(kr), v=torch.zeros_like(v), g=torch.zeros_like(g),
             beta=torch.zeros_like(beta))
    for t in range(T - 1, -1, -1):
        decayed, r, S = kept[t]
        d["q"][:, t] = scale * torch.einsum("bhkv,bhv->bhk", S, do[:, t])
        dS = dS + scale * torch.einsum("bhk,bhv->bhkv", qr[:, t], do[:, t])
        u = beta[:, t, :, None] * r
        du = torch.einsum("bhkv,bhk->bhv", dS, kr[:, t])
        d["beta"][:, t] = (du * r).sum(-1)
        dr = beta[:, t, :, None] * du
        d["v"][:, t] = dr
        d["k"][:, t] = torch.einsum("bhkv,bhv->bhk", dS, u) - torch.einsum("bhkv,bhv->bhk", decayed, dr)
        dS = dS - torch.einsum("bhk,bhv->bhkv", kr[:, t], dr)
        d["g"][:, t] = (dS * decayed).sum((-1, -2))
        dS = dS * torch.exp(g[:, t])[..., None, None]
    for n in ("q", "k"):
        d[n] = d[n].view(B, T, Hk, Hv // Hk, Dk).sum(3)
    d["initial_state"] = dS
    return d
