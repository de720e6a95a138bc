"""The operators of a channels-last token mixer over maps and videos, as they are timed and checked: the gated delta
rule (chunked forward, its gradients, and the recurrent step of serving), rotary positions with several axes, and
group norm with an activation.

A case is a dict of plain values:
    op      "delta"        vmb_delta_rule_fwd: o and, with `state`, the final state from an initial one
            "delta_train"  vmb_delta_rule_fwd keeping its chunk states, and vmb_delta_rule_bwd
            "delta_step"   vmb_delta_rule_step: T tokens a sequence, the state updated in place in a pool of `pool` slots
            "rotary"       vmb_rotary_fwd on q and k (`inverse`: the gradient's direction)
            "norm"         vmb_group_norm_fwd
            "norm_train"   vmb_group_norm_fwd and vmb_group_norm_bwd
    dtype   "f32" or "bf16": storage type of the activations (states, norm weights and statistics are fp32)
    the sizes that each op takes (see `prepare`)

With `own` false the operators are computed in their plain form, elementary torch operations in 32 bits; with `own`
true through the package's entry points.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64  # chunk length of the plain form of the delta rule


def _delta(op, B, T, Hk, Hv, Dk, Dv, dtype, state=False, lens=(), fused=False):
    return dict(op=op, B=B, T=T, Hk=Hk, Hv=Hv, Dk=Dk, Dv=Dv, dtype=dtype, state=state,
                lens=" ".join(str(n) for n in lens), fused=fused)


def _step(B, T, Hk, Hv, Dk, Dv, dtype, pool=0):
    return dict(op="delta_step", B=B, T=T, Hk=Hk, Hv=Hv, Dk=Dk, Dv=Dv, dtype=dtype, pool=pool)


def _rotary(B, axes, Hq, Hk, D, pairs, dtype, positions=False, interleaved=False, inverse=False):
    return dict(op="rotary", B=B, axes=" ".join(str(n) for n in axes), Hq=Hq, Hk=Hk, D=D,
                pairs=" ".join(str(n) for n in pairs), dtype=dtype, positions=positions, interleaved=interleaved,
                inverse=inverse)


def _norm(op, B, H, W, C, G, act, dtype):
    return dict(op=op, B=B, H=H, W=W, C=C, G=G, act=act, dtype=dtype)


def listed():
    # images of a serving batch, of every size from one patch to 64 x 64 patches, packed without padding
    ragged = (1, 3136, 49, 784, 196, 1443, 64, 2809, 4096, 63, 65, 1024, 576, 7, 2025, 961, 128, 333, 3600, 1763, 256, 900,
              15, 1297)
    named = {
        # serving: one stream, one token: launches and latency are all there is
        "step_b1_h6_d64_bf16": _step(1, 1, 6, 6, 64, 64, "bf16"),
        # serving: a full batch of streams in slots of a state pool, two value heads to a key head
        "step_b256_h12_d128_bf16": _step(256, 1, 6, 12, 128, 128, "bf16", pool=320),
        # one 224 x 224 image at the first stage (56 x 56 tokens, 192 channels): three heads, a long sequence
        "delta_b1_t3136_h3_d64": _delta("delta", 1, 3136, 3, 3, 64, 64, "f32", state=True),
        # the same stage of a batch of 32, q, k and v in one projection's output
        "delta_b32_t3136_h3_d64_bf16": _delta("delta", 32, 3136, 3, 3, 64, 64, "bf16", fused=True),
        # prefill of a ragged batch (768 channels) that goes on from earlier states and hands them on
        "delta_packed24_h12_d64_bf16": _delta("delta", len(ragged), 4096, 6, 12, 64, 64, "bf16", True, ragged),
        # segmentation of one 512 x 512 image (128 x 128 tokens): the longest sequence, wide heads
        "delta_b1_t16384_h6_d128_bf16": _delta("delta", 1, 16384, 6, 6, 128, 128, "bf16"),
        # training, second stage (28 x 28 tokens, 384 channels) of a batch of 32
        "train_b32_t784_h6_d64": _delta("delta_train", 32, 784, 6, 6, 64, 64, "f32"),
        # training with wide heads, two value heads to a key head, in bf16: the largest work
        "train_b8_t3136_h12_d128_bf16": _delta("delta_train", 8, 3136, 6, 12, 128, 128, "bf16"),
        # queries and keys of the second stage, rows and columns of the map as positions
        "rotary_b32_28x28_h6_d64": _rotary(32, (28, 28), 6, 6, 64, (16, 16), "f32"),
        # gradients of a video's queries and keys: time, row and column given for each token, part of the head rotated
        "rotary_video_b4_16x28x28_d96_bf16": _rotary(4, (16, 28, 28), 12, 6, 96, (8, 14, 14), "bf16", True, True, True),
        # a segmentation map (128 x 128, 192 channels) on its way into the mixer
        "norm_b8_128x128_c192_bf16": _norm("norm", 8, 128, 128, 192, 8, "silu", "bf16"),
        # training, first stage of a batch of 32
        "norm_train_b32_56x56_c192": _norm("norm_train", 32, 56, 56, 192, 32, "silu", "f32"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(["delta", "delta", "delta", "delta_train", "delta_train", "delta_step", "rotary", "norm",
                     "norm_train"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_train"):
        G = rng.choice([1, 2, 4, 8, 16, 32])
        C = G * _log_int(rng, max(1, 32 // G), max(2, 1536 // G))
        H, W = (_log_int(rng, 5, 128), _log_int(rng, 5, 128)) if rng.random() < 0.5 else (rng.choice([7, 14, 28, 56, 128]),) * 2
        most = 20_000_000 if op == "norm" else 12_000_000
        B = min(_log_int(rng, 1, 64), max(1, most // (H * W * C)))
        if B * H * W * C > most:
            H, W = 28, 28
        return _norm(op, B, H, W, C, G, rng.choice(["none", "silu", "silu", "gelu"]), dtype)
    if op == "rotary":
        n = rng.choice([1, 2, 2, 3])
        axes = [_log_int(rng, 4, 4096)] if n == 1 else [_log_int(rng, 5, 64) for _ in range(2)]
        if n == 3:
            axes = [rng.randint(2, 16)] + [_log_int(rng, 5, 32) for _ in range(2)]
        pairs = [rng.randint(1, 24) for _ in range(n)]
        D = rng.choice([2 * sum(pairs), 2 * sum(pairs) + rng.randint(1, 32), 8 * ((2 * sum(pairs) + 15) // 8)])
        Hk = rng.choice([1, 2, 3, 4, 6])
        Hq = Hk * rng.choice([1, 2, 3])
        B = min(_log_int(rng, 1, 32), max(1, 20_000_000 // (math.prod(axes) * D * (Hq + Hk))))
        return _rotary(B, axes, Hq, Hk, D, pairs, dtype, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)
    Dk = rng.choice([64, 64, 128, 128, 32, 48, rng.randint(9, 127)])
    Dv = rng.choice([Dk, Dk, 64, 128, rng.randint(9, 160)])
    Hk = rng.choice([1, 2, 3, 4, 6])
    Hv = Hk * rng.choice([1, 1, 2, 3])
    if op == "delta_step":
        B = min(_log_int(rng, 1, 256), max(1, 50_000_000 // (Hv * Dk * Dv)))
        return _step(B, rng.choice([1, 1, 1, 2, 4, 7]), Hk, Hv, Dk, Dv, dtype, rng.choice([0, B + rng.randint(1, 40)]))
    most = (30_000_000 if op == "delta" else 14_000_000) // (Hv * max(Dk, Dv))
    short = 1 if op == "delta" else 2  # (one token alone leaves no gradient of g)
    T = min(_log_int(rng, short, 16384), most) if rng.random() < 0.6 else min(rng.choice([49, 196, 784, 3136, 16384]), most)
    B = min(_log_int(rng, 1, 64), max(1, most // T))
    lens = [rng.randint(0, 3) + _log_int(rng, short, max(2, T - 3)) for _ in range(B)] if rng.random() < 0.3 and T > 8 else []
    if lens:
        T = max(lens)
    return _delta(op, B, T, Hk, Hv, Dk, Dv, dtype, op == "delta" and rng.random() < 0.5, lens, rng.random() < 0.3)


def _ints(text):
    return [int(n) for n in text.split()]


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(shape, device="cuda", generator=gen)

    dt, st = DTYPES[case["dtype"]], {"case": case}
    if case["op"].startswith("delta"):
        return _prepare_delta(case, st, dt, normal, uniform, gen)
    if case["op"] == "rotary":
        B, axes, pairs, D = case["B"], _ints(case["axes"]), _ints(case["pairs"]), case["D"]
        T = math.prod(axes)
        st["q"], st["k"] = normal(B, T, case["Hq"], D).to(dt), normal(B, T, case["Hk"], D).to(dt)
        # each axis has its own frequencies, 1 down to about 1/100 (positions are rows and columns of a map) or 1/10000
        base = 100.0 if len(axes) > 1 else 10000.0
        st["freq"] = torch.cat([base ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n) for n in pairs]).float()
        st["sections"], st["grid"], st["positions"] = tuple(pairs), tuple(axes), None
        if case["positions"]:  # tokens at places of their own: crops of a larger map, frames from some second on
            at = torch.cartesian_prod(*[torch.arange(n, device="cuda") for n in axes]).view(T, len(axes)).t()
            shift = torch.randint(0, 64, (len(axes), B, 1), device="cuda", generator=gen)
            st["positions"] = (at.unsqueeze(1) + shift).to(torch.int32).contiguous()
            st["grid"] = None
        return st
    B, H, W, C = case["B"], case["H"], case["W"], case["C"]
    # a map whose channels have means and scales of their own
    st["x"] = ((0.3 + uniform(1, 1, 1, C)) * normal(B, H, W, C) + 0.5 * normal(B, 1, 1, C)).to(dt)
    st["weight"], st["bias"] = 0.75 + 0.5 * uniform(C), 0.2 * normal(C)
    if case["op"] == "norm_train":
        st["dy"] = normal(B, H, W, C).to(dt)
    return st


def _prepare_delta(case, st, dt, normal, uniform, gen):
    """Keys and queries of length one around a direction that a head's tokens share, a step weight beta = sigmoid, and
    a log decay g = -a dt with a per head in [1, 16] and dt log-uniform in [1e-3, 0.1]."""
    B, T, Hk, Hv, Dk, Dv = (case[n] for n in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
    lens = _ints(case.get("lens", ""))
    b, t = (1, sum(lens)) if lens else (B, T)

    def unit(x):
        return x / x.square().sum(-1, keepdim=True).sqrt()

    q, k = (unit(normal(b, t, Hk, Dk) + 0.5 * normal(1, 1, Hk, Dk)) for _ in range(2))
    v = normal(b, t, Hv, Dv)
    if case.get("fused"):  # as one projection writes them: the heads of q, k and v side by side in a token's row
        row = torch.cat([x.reshape(b, t, -1) for x in (q, k, v)], -1).to(dt)
        q, k, v = (x.view(b, t, h, -1) for x, h in zip(row.split([Hk * Dk, Hk * Dk, Hv * Dv], -1), (Hk, Hk, Hv)))
    else:
        q, k, v = q.to(dt), k.to(dt), v.to(dt)
    st["q"], st["k"], st["v"] = q, k, v
    st["g"] = (-(1 + 15 * uniform(Hv)) * torch.exp(math.log(1e-3) + math.log(100.0) * uniform(b, t, Hv))).to(dt)
    st["beta"] = torch.sigmoid(normal(b, t, Hv)).to(dt)
    st["initial"] = None
    if case["op"] == "delta_step":
        pool = case["pool"] or B
        st["state"], st["slots"] = normal(pool, Hv, Dk, Dv) * 0.3, None
        if case["pool"]:  # slots in no order; every 16th row of the batch is padding
            slots = torch.randperm(pool, device="cuda", generator=gen)[:B].to(torch.int32)
            slots[15::16] = -1
            st["slots"] = slots
        return st
    if case["state"]:
        st["initial"] = normal(B, Hv, Dk, Dv) * 0.3
    st["offsets"], st["lens"] = None, lens
    if lens:
        st["offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    if case["op"] == "delta_train":
        st["do"] = normal(b, t, Hv, Dv).to(dt)
    return st


# ------------------------------------------------------------------ one pass


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        import paper_2412_16602_gb300 as vmb

        if op in ("delta", "delta_train"):
            packed = dict(offsets=st["offsets"], max_len=case["T"]) if st["lens"] else {}
            o, final, saved = vmb.vmb_delta_rule_fwd(st["q"], st["k"], st["v"], st["g"], st["beta"],
                                                     initial_state=st["initial"], want_state=case["state"],
                                                     want_saved=op == "delta_train", **packed)
            if op == "delta":
                return (o, final) if case["state"] else o
            d = vmb.vmb_delta_rule_bwd(st["q"], st["k"], st["v"], st["g"], st["beta"], st["do"], saved, **packed)
            return o, d["q"], d["k"], d["v"], d["g"], d["beta"]
        if op == "delta_step":
            o = vmb.vmb_delta_rule_step(st["q"], st["k"], st["v"], st["g"], st["beta"], st["state"], slots=st["slots"])
            return o, st["state"]
        if op == "rotary":
            return vmb.vmb_rotary_fwd(st["q"], st["k"], st["freq"], st["positions"], sections=st["sections"],
                                      grid=st["grid"], interleaved=case["interleaved"], inverse=case["inverse"])
        if op == "norm":
            return vmb.vmb_group_norm_fwd(st["x"], st["weight"], st["bias"], case["G"], act=case["act"])[0]
        y, stats = vmb.vmb_group_norm_fwd(st["x"], st["weight"], st["bias"], case["G"], act=case["act"], want_stats=True)
        d = vmb.vmb_group_norm_bwd(st["x"], st["weight"], st["bias"], stats, st["dy"], case["G"], act=case["act"])
        return y, d["x"], d["weight"], d["bias"]
    if op in ("delta", "delta_train"):
        return _plain_delta(st, case)
    if op == "delta_step":
        return _plain_step(st, case)
    if op == "rotary":
        return _plain_rotary(st, case)
    return _plain_norm(st, case)


# ------------------------------------------------------------------ the plain forms


def _padded(x, lens):
    """[1, sum(lens), ...] -> [len(lens), max(lens), ...], zeros behind each sequence."""
    out = x.new_zeros(len(lens), max(max(lens), 1), *x.shape[2:])
    for i, s in enumerate(torch.split(x[0], lens)):
        out[i, :lens[i]] = s
    return out


def _packed(x, lens):
    return torch.cat([x[i, :n] for i, n in enumerate(lens)]).unsqueeze(0)


def _chunks(x, heads):
    """[B, T, h, d] -> fp32 [B, heads, chunks, CHUNK, d], zeros behind the last token, shared heads repeated."""
    B, T, h, d = x.shape
    n = (T + CHUNK - 1) // CHUNK
    y = x.new_zeros(B, n * CHUNK, h, d, dtype=torch.float32)
    y[:, :T] = x
    y = y.view(B, n, CHUNK, h, d).permute(0, 3, 1, 2, 4)
    return y.repeat_interleave(heads // h, 1)


def _tokens(y, T):
    B, h, n, c, d = y.shape
    return y.permute(0, 2, 3, 1, 4).reshape(B, n * c, h, d)[:, :T]


def _plain_delta(st, case):
    """The chunked form.  In a chunk with cumulative log decays c and start state S (Dk x Dv):
    A_ij = beta_i e^(c_i - c_j) k_i.k_j (j < i), U = (I + A)^-1 beta (V - e^c K S),
    O = scale (e^c Q S + (e^(c_i - c_j) q_i.k_j, j <= i) U), S' = e^c_last S + sum_j e^(c_last - c_j) k_j U_j^T."""
    lens, Hv, Hk = st["lens"], case["Hv"], case["Hk"]
    ins = [st[n] for n in ("q", "k", "v")] + [st[n].unsqueeze(-1) for n in ("g", "beta")]
    if lens:
        ins = [_padded(x, lens) for x in ins]
    B, T = ins[0].shape[:2]
    q, k, v, g, beta = (_chunks(x, Hv) for x in ins)
    scale, dt = case["Dk"] ** -0.5, st["q"].dtype
    n = q.shape[2]
    c = g.cumsum(3)
    low = torch.tril(torch.ones(CHUNK, CHUNK, device=q.device, dtype=torch.bool))
    decay = torch.exp(torch.where(low, c - c.transpose(3, 4), -math.inf))
    strict = torch.tril(decay, -1)
    A = beta * strict * (k @ k.transpose(3, 4))
    P = scale * decay * (q @ k.transpose(3, 4))
    inv = torch.eye(CHUNK, device=q.device).expand_as(A).clone()
    for i in range(1, CHUNK):
        inv[..., i, :] -= (A[..., i, None, :i] @ inv[..., :i, :]).squeeze(-2)
    ec, last = torch.exp(c), c[..., -1:, :]
    tail, elast = torch.exp(last - c), torch.exp(last)
    qd, kt, kd = scale * ec * q, tail * k, ec * k
    S = torch.zeros(B, Hv, case["Dk"], case["Dv"], device=q.device) if st["initial"] is None else st["initial"]
    starts, Us, Rs, os = [], [], [], []
    for i in range(n):
        R = v[:, :, i] - kd[:, :, i] @ S
        U = inv[:, :, i] @ (beta[:, :, i] * R)
        os.append(qd[:, :, i] @ S + P[:, :, i] @ U)
        starts.append(S), Us.append(U), Rs.append(R)
        S = elast[:, :, i] * S + kt[:, :, i].transpose(2, 3) @ U

    def back(x, heads=Hv):
        x = _tokens(x, T)
        if heads != Hv:
            x = x.reshape(B, T, heads, Hv // heads, -1).sum(3)
        return (_packed(x, lens) if lens else x).to(dt)

    o = back(torch.stack(os, 2))
    if case["op"] == "delta":
        return (o, S) if case["state"] else o
    # the gradients: dU and dS from chunk to chunk in reverse, the others for all chunks at once
    do = _chunks(_padded(st["do"], lens) if lens else st["do"], Hv)
    dS, dSs, dXs = torch.zeros_like(S), [None] * n, [None] * n
    for i in range(n - 1, -1, -1):
        dSs[i] = dS
        dU = P[:, :, i].transpose(2, 3) @ do[:, :, i] + kt[:, :, i] @ dS
        dXs[i] = inv[:, :, i].transpose(2, 3) @ dU
        dS = elast[:, :, i] * dS + qd[:, :, i].transpose(2, 3) @ do[:, :, i] \
            - kd[:, :, i].transpose(2, 3) @ (beta[:, :, i] * dXs[i])
    S, dS, U, R, dX = (torch.stack(x, 2) for x in (starts, dSs, Us, Rs, dXs))
    dR = beta * dX
    dA = -(dR @ U.transpose(3, 4)) * strict  # times k_i.k_j's gradient: beta is in dR
    dP = scale * (do @ U.transpose(3, 4)) * decay
    dq = scale * ec * (do @ S.transpose(3, 4)) + dP @ k
    dk_row = dA @ k - ec * (dR @ S.transpose(3, 4))
    dk_tail = tail * (U @ dS.transpose(3, 4))
    dk_col = dA.transpose(3, 4) @ k + dP.transpose(3, 4) @ q + dk_tail
    E = strict * (k @ k.transpose(3, 4))
    dbeta = (dX * (R - E @ U)).sum(-1, keepdim=True)
    dc = (q * dq).sum(-1, keepdim=True) + (k * (dk_row - dk_col)).sum(-1, keepdim=True)
    dc[..., -1:, :] += (k * dk_tail).sum((3, 4), keepdim=True) + elast * (S * dS).sum((3, 4), keepdim=True)
    dg = dc.flip(3).cumsum(3).flip(3)
    return (o, back(dq, Hk), back(dk_row + dk_col, Hk), back(dR), back(dg).squeeze(-1), back(dbeta).squeeze(-1))


def _plain_step(st, case):
    B, T, r = case["B"], case["T"], case["Hv"] // case["Hk"]
    q, k = (st[n].float().repeat_interleave(r, 2) for n in ("q", "k"))
    v, g, beta = (st[n].float() for n in ("v", "g", "beta"))
    slots = torch.arange(B, device=q.device) if st["slots"] is None else st["slots"].long()
    used = slots >= 0
    S = st["state"][slots.clamp(min=0)]
    os = []
    for t in range(T):
        S = torch.exp(g[:, t])[..., None, None] * S
        u = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, :, :, None]).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None]
        os.append((S * q[:, t, :, :, None]).sum(2) * case["Dk"] ** -0.5)
    o = torch.stack(os, 1) * used.view(B, 1, 1, 1)
    st["state"][slots[used]] = S[used]
    return o.to(st["q"].dtype), st["state"]


def _angles(st, case, dtype):
    """Angles [B or 1, T, 1, pairs] of every token, from its position on each axis."""
    pairs = st["sections"]
    if st["positions"] is None:
        at = torch.cartesian_prod(*[torch.arange(n, device="cuda") for n in st["grid"]]).view(-1, len(pairs)).t().unsqueeze(1)
    else:
        at = st["positions"]
    axis = torch.repeat_interleave(torch.arange(len(pairs), device="cuda"), torch.tensor(pairs, device="cuda"))
    return (at.to(dtype)[axis].permute(1, 2, 0) * st["freq"].to(dtype)).unsqueeze(2)


def _plain_rotary(st, case):
    a = _angles(st, case, torch.float32)
    cos, sin = torch.cos(a), -torch.sin(a) if case["inverse"] else torch.sin(a)
    P = a.shape[-1]

    def turn(x):
        y = x.float()
        first, second = (y[..., 0:2 * P:2], y[..., 1:2 * P:2]) if case["interleaved"] else (y[..., :P], y[..., P:2 * P])
        one, two = first * cos - second * sin, second * cos + first * sin
        both = torch.stack([one, two], -1).flatten(-2) if case["interleaved"] else torch.cat([one, two], -1)
        return torch.cat([both, y[..., 2 * P:]], -1).to(x.dtype)

    return turn(st["q"]), turn(st["k"])


def _activation(z, act):
    """act(z) and act'(z)."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def _plain_norm(st, case):
    B, G, C, dt = case["B"], case["G"], case["C"], st["x"].dtype
    x = st["x"].float().view(B, -1, G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean((1, 3), keepdim=True) + 1e-5)
    n = (x - mean) * rstd
    w = st["weight"].view(G, C // G)
    y, slope = _activation(n * w + st["bias"].view(G, C // G), case["act"])
    y = y.reshape(st["x"].shape).to(dt)
    if case["op"] == "norm":
        return y
    dz = st["dy"].float().view(x.shape) * slope
    dn = dz * w
    dx = rstd * (dn - dn.mean((1, 3), keepdim=True) - n * (dn * n).mean((1, 3), keepdim=True))
    return y, dx.reshape(st["x"].shape).to(dt), (dz * n).sum((0, 1)).reshape(C), dz.sum((0, 1)).reshape(C)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    s = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op.startswith("delta"):
        B, T, Hk, Hv, Dk, Dv = (case[n] for n in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
        tokens = sum(_ints(case["lens"])) if case.get("lens") else B * T
        qkv, o, gates, state = tokens * (2 * Hk * Dk + Hv * Dv), tokens * Hv * Dv, 2 * tokens * Hv, B * Hv * Dk * Dv
        # per token and head: decay the state, S^T k, the rank-one update, S^T q
        flops = 7 * tokens * Hv * Dk * Dv
        if op == "delta_step":
            rows = B - (B // 16 if case["pool"] else 0)
            return {"bytes": s * (qkv + o + gates) + 8 * (state // B) * rows, "flops": flops // B * rows}
        if op == "delta":
            return {"bytes": s * (qkv + o + gates) + (8 * state if case["state"] else 0), "flops": flops}
        # the gradients read the inputs and do, write one gradient for each input, and take the recurrence's reverse
        return {"bytes": s * (2 * qkv + 2 * o + 2 * gates), "flops": flops + 15 * tokens * Hv * Dk * Dv}
    if op == "rotary":
        T, P = math.prod(_ints(case["axes"])), sum(_ints(case["pairs"]))
        values = case["B"] * T * (case["Hq"] + case["Hk"]) * case["D"]
        place = 4 * len(_ints(case["axes"])) * case["B"] * T if case["positions"] else 0
        return {"bytes": 2 * s * values + place + 4 * P, "flops": 6 * case["B"] * T * (case["Hq"] + case["Hk"]) * P}
    values = case["B"] * case["H"] * case["W"] * case["C"]
    if op == "norm":
        return {"bytes": 2 * s * values + 8 * case["C"], "flops": 12 * values}
    return {"bytes": 4 * s * values + 16 * case["C"], "flops": 36 * values}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("delta", "delta_train"):
        return _exact_delta(st, case)
    if case["op"] == "delta_step":
        B, r = case["B"], case["Hv"] // case["Hk"]
        slots = list(range(B)) if st["slots"] is None else st["slots"].tolist()
        state, o = st["state"].double(), torch.zeros(B, case["T"], case["Hv"], case["Dv"], dtype=torch.float64, device="cuda")
        rows = [b for b in range(B) if slots[b] >= 0]
        at = [slots[b] for b in rows]
        S = state[at]
        for t in range(case["T"]):
            q, k = (st[n][rows, t].double().repeat_interleave(r, 1) for n in ("q", "k"))
            S, out = _token(S, q, k, *(st[n][rows, t].double() for n in ("v", "g", "beta")))[:2]
            o[rows, t] = out * case["Dk"] ** -0.5
        state[at] = S
        return o, state
    if case["op"] == "rotary":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), _angles(st, case, torch.float64))
        turn = turn.conj() if case["inverse"] else turn
        P = turn.shape[-1]
        out = []
        for name in ("q", "k"):
            x = st[name].double()
            if case["interleaved"]:
                z = torch.view_as_complex(x[..., :2 * P].unflatten(-1, (P, 2)).contiguous()) * turn
                both = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(x[..., :P], x[..., P:2 * P]) * turn
                both = torch.cat([z.real, z.imag], -1)
            out.append(torch.cat([both, x[..., 2 * P:]], -1))
        return tuple(out)
    return _exact_norm(st, case)


def _token(S, q, k, v, g, beta):
    """One token of the recurrence: the state after it, S^T q, the decayed state before it, the residual."""
    S = S * torch.exp(g)[..., None, None]
    r = v - torch.einsum("bhkv,bhk->bhv", S, k)
    return (N := S + torch.einsum("bhk,bhv->bhkv", k, beta[..., None] * r)), torch.einsum("bhkv,bhk->bhv", N, q), S, r


def _exact_delta(st, case):
    """Token after token; the gradients by the reverse recurrence, states recomputed in stretches of 64 tokens."""
    lens, Hk, Hv, Dk, Dv = st["lens"], case["Hk"], case["Hv"], case["Dk"], case["Dv"]
    r, scale = Hv // Hk, Dk ** -0.5
    names = ["q", "k", "v", "g", "beta"] + (["do"] if case["op"] == "delta_train" else [])
    x = {n: (_padded(st[n], lens) if lens else st[n]).double() for n in names}
    B, T = x["q"].shape[:2]
    if case["op"] == "delta" and T * B * Hv * Dk * Dv > 4e10:
        return None
    if case["op"] == "delta_train" and T * B * Hv * Dk * Dv > 1.3e10:
        return None
    for n in ("q", "k"):
        x[n] = x[n].repeat_interleave(r, 2)
    at = {n: x[n].transpose(0, 1).contiguous() for n in names}
    S = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64, device="cuda") if st["initial"] is None else st["initial"].double()
    o = torch.empty(T, B, Hv, Dv, dtype=torch.float64, device="cuda")
    kept = []
    for t in range(T):
        if t % 64 == 0:
            kept.append(S)
        S, o[t] = _token(S, *(at[n][t] for n in names[:5]))[:2]

    def back(y):
        y = y.transpose(0, 1)
        return _packed(y, lens) if lens else y

    o *= scale
    if case["op"] == "delta":
        return (back(o), S) if case["state"] else back(o)
    d = {n: torch.empty_like(at[n]) for n in names[:5]}
    dS = torch.zeros_like(S)
    for j in range(len(kept) - 1, -1, -1):
        S, seen = kept[j], []
        for t in range(64 * j, min(T, 64 * j + 64)):
            N, _, decayed, res = _token(S, *(at[n][t] for n in names[:5]))
            seen.append((S, N, decayed, res))
            S = N
        for t in range(min(T, 64 * j + 64) - 1, 64 * j - 1, -1):
            before, N, decayed, res = seen[t - 64 * j]
            q, k, g, beta, do = (at[n][t] for n in ("q", "k", "g", "beta", "do"))
            d["q"][t] = scale * torch.einsum("bhkv,bhv->bhk", N, do)
            dS = dS + scale * torch.einsum("bhk,bhv->bhkv", q, do)
            du = torch.einsum("bhkv,bhk->bhv", dS, k)
            d["beta"][t] = (du * res).sum(-1)
            dr = beta[..., None] * du
            d["v"][t] = dr
            d["k"][t] = torch.einsum("bhkv,bhv->bhk", dS, beta[..., None] * res) - torch.einsum("bhkv,bhv->bhk", decayed, dr)
            dS = dS - torch.einsum("bhk,bhv->bhkv", k, dr)
            d["g"][t] = (dS * decayed).sum((2, 3))
            dS = dS * torch.exp(g)[..., None, None]
        seen.clear()
    shared = [back(d[n]) for n in ("q", "k")]
    shared = [y.reshape(*y.shape[:2], Hk, r, Dk).sum(3) for y in shared]
    return (back(o), *shared, back(d["v"]), back(d["g"]), back(d["beta"]))


def _exact_norm(st, case):
    """Group after group of channels; the gradient as the derivative's rows, not through the plain form's names."""
    x, w, b = st["x"].double(), st["weight"].double(), st["bias"].double()
    m, train = case["C"] // case["G"], case["op"] == "norm_train"
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.empty_like(w), torch.empty_like(b)
    for j in range(case["G"]):
        at = slice(j * m, (j + 1) * m)
        xs = x[..., at]
        var, mean = torch.var_mean(xs, dim=(1, 2, 3), correction=0, keepdim=True)
        sd = torch.sqrt(var + 1e-5)
        n = (xs - mean) / sd
        z = torch.addcmul(b[at], n, w[at])
        if case["act"] == "silu":
            s = torch.sigmoid(z)
            y[..., at], slope = z * s, s + z * s * torch.sigmoid(-z)
        elif case["act"] == "gelu":
            cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
            y[..., at], slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            y[..., at], slope = z, torch.ones_like(z)
        if train:
            dz = st["dy"][..., at].double() * slope
            dw[at], db[at] = (dz * n).sum((0, 1, 2)), dz.sum((0, 1, 2))
            dn = dz * w[at]
            dx[..., at] = (dn - dn.mean((1, 2, 3), keepdim=True) - n * (dn * n).mean((1, 2, 3), keepdim=True)) / sd
    return (y, dx, dw, db) if train else y
