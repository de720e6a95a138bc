"""The operators of a layer around the selective scan for sequences of tokens, channels last, as they are timed and
checked: the short causal convolution and the selective state space scan with its gate (prompts, gradients, single
tokens), root-mean-square norm with the residual's addition and an output in 8 bits, and the matrix product with bias,
activation and residual.

A case is a dict of plain values:
    op      "conv"         vmb_causal_conv_fwd (`state`: from initial states, and the states after each sequence)
            "conv_train"   vmb_causal_conv_fwd and vmb_causal_conv_bwd
            "conv_step"    vmb_causal_conv_step: T tokens a stream, the inputs kept in slots of a pool
            "scan"         vmb_token_scan_fwd
            "scan_train"   vmb_token_scan_fwd keeping its chunk states, and vmb_token_scan_bwd
            "scan_step"    vmb_token_scan_step
            "norm"         vmb_rms_norm_fwd with the residual's addition
            "norm8"        the same with an output in 8 bits and one scale a row
            "norm_train"   vmb_rms_norm_fwd and vmb_rms_norm_bwd
            "linear"       vmb_linear_fwd of bf16
            "linear8"      vmb_linear_fwd of 8-bit values with scales
            "linear_grad"  vmb_linear_bwd
    dtype   "f32" or "bf16": storage type of the activations (states of the scan, norm weights, biases, A and D are fp32)
    the sizes that each op takes (see `prepare`)

With `own` false the operators are computed in their plain form, elementary torch operations in 32 bits; with `own`
true through the package's entry points.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def _conv(op, B, T, C, W, act, dtype, state=False, lens=(), half=False):
    return dict(op=op, B=B, T=T, C=C, W=W, act=act, dtype=dtype, state=state, lens=" ".join(str(n) for n in lens),
                half=half)


def _conv_step(B, T, C, W, act, dtype, pool=0):
    return dict(op="conv_step", B=B, T=T, C=C, W=W, act=act, dtype=dtype, pool=pool)


def _scan(op, B, T, D, N, dtype, gate=False, state=False, lens=(), half=False):
    return dict(op=op, B=B, T=T, D=D, N=N, dtype=dtype, gate=gate, state=state, lens=" ".join(str(n) for n in lens),
                half=half)


def _scan_step(B, T, D, N, dtype, gate=True, pool=0):
    return dict(op="scan_step", B=B, T=T, D=D, N=N, dtype=dtype, gate=gate, pool=pool)


def _norm(op, rows, C, dtype, residual=True):
    return dict(op=op, rows=rows, C=C, dtype=dtype, residual=residual)


def _linear(op, M, K, N, act="none", bias=True, residual=False):
    return dict(op=op, M=M, K=K, N=N, act=act, bias=bias, residual=residual, dtype="bf16")


def listed():
    # prompts of a serving batch, of every length from one token to 4096, packed without padding
    ragged = (1, 3136, 49, 784, 196, 1443, 64, 2809, 4096, 63, 65, 1024, 576, 7, 2025, 961, 128, 333, 3600, 1763, 256, 900,
              15, 1297)
    named = {
        # serving: one token of each of 64 streams, their last inputs in slots of a pool: launches and latency
        "conv_step_b64_c2048_bf16": _conv_step(64, 1, 2048, 4, "silu", "bf16", pool=80),
        # prefill of a ragged batch that goes on from earlier tokens; x is one half of a projection's output
        "conv_packed24_c1536_bf16": _conv("conv", len(ragged), 4096, 1536, 4, "silu", "bf16", True, ragged, True),
        # training: a batch of sequences, three taps
        "conv_train_b8_t3136_c768": _conv("conv_train", 8, 3136, 768, 3, "silu", "f32"),
        # serving: a full batch of streams in slots of a state pool
        "scan_step_b256_d2048_n16_bf16": _scan_step(256, 1, 2048, 16, "bf16", True, 320),
        # one 224 x 224 image as a sequence (second stage's channels, first stage's tokens): few channels, a long chain
        "scan_b1_t3136_d384_n16": _scan("scan", 1, 3136, 384, 16, "f32"),
        # prefill of the ragged batch with the gate, from earlier states and handing them on
        "scan_packed24_d1536_n16_bf16": _scan("scan", len(ragged), 4096, 1536, 16, "bf16", True, True, ragged, True),
        # training with the gate in bf16
        "scan_train_b4_t2048_d2048_n16_bf16": _scan("scan_train", 4, 2048, 2048, 16, "bf16", True),
        # the norm before an 8-bit projection, residual added
        "norm8_16384x1536_bf16": _norm("norm8", 16384, 1536, "bf16"),
        # training, 32 maps of 28 x 28 tokens
        "norm_train_25088x768": _norm("norm_train", 25088, 768, "f32"),
        # serving: the projection of one token back to the residual stream: every weight is read once
        "linear_1x2048x4096_bf16": _linear("linear", 1, 2048, 4096, residual=True),
        # the wide projection of a long prompt in 8 bits, GELU
        "linear8_16384x1536x6144": _linear("linear8", 16384, 1536, 6144, "gelu"),
        # gradients of a projection with SiLU
        "linear_grad_8192x1024x4096_bf16": _linear("linear_grad", 8192, 1024, 4096, "silu"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lengths(rng, B, T):
    return [rng.randint(0, 2) + _log_int(rng, 1, max(2, T - 2)) for _ in range(B)]


def draw(rng):
    """One more case: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(["conv", "conv_train", "conv_step", "scan", "scan", "scan_train", "scan_train", "scan_step", "norm",
                     "norm8", "norm_train", "linear", "linear", "linear8", "linear_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if op.startswith("norm"):
        C = rng.choice([96, 192, 384, 768, 1024, 1536, 2048, 4096, _log_int(rng, 8, 6000), _log_int(rng, 8, 6000)])
        return _norm(op, min(_log_int(rng, 1, 30000), 19_000_000 // C), C, dtype, rng.random() < 0.7)
    if op.startswith("linear"):
        M = rng.choice([_log_int(rng, 1, 16), _log_int(rng, 1, 16384), _log_int(rng, 100, 16384)])
        K, N = 16 * _log_int(rng, 4, 256), 8 * _log_int(rng, 8, 512)
        if op != "linear_grad" and rng.random() < 0.3:
            N = N + rng.randint(1, 7)
        if op != "linear8" and rng.random() < 0.3:
            K = K + 8
        most = {"linear": 6e10, "linear8": 1.2e11, "linear_grad": 3e10}[op]
        return _linear(op, min(M, max(1, int(most / K / N))), K, N, rng.choice(["none", "silu", "gelu"]), rng.random() < 0.6,
                       op != "linear_grad" and rng.random() < 0.5)
    C = rng.choice([96, 192, 384, 768, 1024, 1536, 2048, _log_int(rng, 20, 4096), _log_int(rng, 20, 4096)])
    W, N, act = rng.choice([2, 3, 4, 4]), rng.choice([16, 16, 16, 8, 4, rng.randint(1, 16)]), rng.choice(["silu", "silu", "none"])
    if op.endswith("_step"):
        B = min(_log_int(rng, 1, 256), 1_000_000 // C)
        T, pool = rng.choice([1, 1, 1, 2, 3, 5]), rng.choice([0, B + rng.randint(1, 40)])
        return _conv_step(B, T, C, W, act, dtype, pool) if op == "conv_step" else _scan_step(B, T, C, N, dtype, rng.random() < 0.7, pool)
    most = {"conv": 38_000_000, "conv_train": 18_000_000, "scan": 38_000_000, "scan_train": 16_000_000}[op] // C
    T = min(_log_int(rng, 1, 16384), most) if rng.random() < 0.6 else min(rng.choice([49, 196, 784, 2048, 3136, 16384]), most)
    B = min(_log_int(rng, 1, 64), max(1, most // T))
    lens = _lengths(rng, B, T) if rng.random() < 0.35 and T > 8 else []
    if sum(lens) > most:
        lens = []
    if lens:
        T = max(lens)
    state, half = not op.endswith("train") and rng.random() < 0.5, rng.random() < 0.4
    if op.startswith("conv"):
        return _conv(op, B, T, C, W, act, dtype, state, lens, half)
    return _scan(op, B, T, C, N, dtype, rng.random() < 0.7, state, lens, half)


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
    if case["op"].startswith("norm"):
        rows, C = case["rows"], case["C"]
        # a branch's output and a residual stream whose channels have scales of their own
        st["x"], st["weight"] = normal(rows, C).to(dt), 0.75 + 0.5 * uniform(C)
        st["residual"] = (3 * (0.1 + uniform(C)) * normal(rows, C)).to(dt) if case["residual"] else None
        if case["op"] == "norm_train":
            st["dy"], st["dsum"] = normal(rows, C).to(dt), normal(rows, C).to(dt)
        return st
    if case["op"].startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        x, w = normal(M, K), normal(N, K) / math.sqrt(K)
        if case["op"] == "linear8":  # one scale for each row of x and of the weights
            for n, t in (("x", x), ("weight", w)):
                scale = t.abs().amax(1, keepdim=True) / 448
                st[n], st[n + "_scale"] = (t / scale).to(torch.float8_e4m3fn), scale.view(-1)
        else:
            st["x"], st["weight"] = x.to(dt), w.to(dt)
        st["bias"] = 0.3 * normal(N) if case["bias"] else None
        st["residual"] = normal(M, N).to(dt) if case["residual"] else None
        if case["op"] == "linear_grad":
            st["dy"], st["pre"] = normal(M, N).to(dt), normal(M, N).to(dt) if case["act"] != "none" else None
        return st
    B, T = case["B"], case["T"]
    lens = _ints(case.get("lens", ""))
    b, t = (1, sum(lens)) if lens else (B, T)
    C = case.get("C") or case["D"]
    st["offsets"] = None
    if lens:
        st["offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")

    def halves(*parts):
        """Side by side in a token's row, as one projection writes them, or each dense."""
        if not case.get("half"):
            return [p.to(dt) for p in parts]
        return torch.cat(parts, -1).to(dt).split([p.shape[-1] for p in parts], -1)

    pool = case.get("pool") or B
    if case["op"].endswith("_step"):
        st["slots"] = None
        if case["pool"]:  # slots in no order; every 16th row of the batch is padding
            slots = torch.randperm(pool, device="cuda", generator=gen)[:B].to(torch.int32)
            slots[15::16] = -1
            st["slots"] = slots
    if case["op"].startswith("conv"):
        W = case["W"]
        st["x"] = halves(normal(b, t, C), normal(b, t, C if case.get("half") else 0))[0]
        st["weight"], st["bias"] = (2 * uniform(C, W) - 1) / math.sqrt(W), 0.2 * normal(C)
        if case["op"] == "conv_step":
            st["state"] = normal(pool, W - 1, C).to(dt)
            return st
        st["initial"] = normal(B, W - 1, C).to(dt) if case["state"] else None
        if case["op"] == "conv_train":
            st["dy"] = normal(b, t, C).to(dt)
        return st
    N = case["N"]
    # x as the convolution's SiLU leaves it; step sizes softplus(delta + bias) around 1e-3 .. 0.1; A = -1 .. -N and around
    x = normal(b, t, C)
    x, z = halves(x / (1 + torch.exp(-x)), normal(b, t, C) if case["gate"] else normal(b, t, 0))
    st["x"], st["z"] = x, z if case["gate"] else None
    st["delta"] = (0.5 * normal(b, t, C)).to(dt)
    st["Bm"], st["Cm"] = halves(normal(b, t, N), normal(b, t, N))
    step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(C))
    st["bias"] = step + torch.log(-torch.expm1(-step))
    st["A"] = -torch.arange(1, N + 1, device="cuda") * (0.75 + 0.5 * uniform(C, N))
    st["D"] = 0.5 + uniform(C)
    if case["op"] == "scan_step":
        st["state"] = 0.3 * normal(pool, C, N)
        return st
    st["initial"] = 0.3 * normal(B, C, N) if case["state"] else None
    if case["op"] == "scan_train":
        st["dy"] = normal(b, t, C).to(dt)
    return st


# ------------------------------------------------------------------ one pass


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        import paper_2412_16602_gb300 as vmb

        if op == "conv":
            y, last = vmb.vmb_causal_conv_fwd(st["x"], st["weight"], st["bias"], act=case["act"], initial_state=st["initial"],
                                              offsets=st["offsets"], want_state=case["state"])
            return (y, last) if case["state"] else y
        if op == "conv_train":
            y, _ = vmb.vmb_causal_conv_fwd(st["x"], st["weight"], st["bias"], act=case["act"], offsets=st["offsets"])
            d = vmb.vmb_causal_conv_bwd(st["x"], st["weight"], st["bias"], st["dy"], act=case["act"], offsets=st["offsets"])
            return y, d["x"], d["weight"], d["bias"]
        if op == "conv_step":
            y = vmb.vmb_causal_conv_step(st["x"], st["weight"], st["bias"], st["state"], act=case["act"], slots=st["slots"])
            return y, st["state"]
        if op.startswith("scan"):
            ins = [st[n] for n in ("x", "delta", "A", "Bm", "Cm", "D", "bias", "z")]
            if op == "scan_step":
                return vmb.vmb_token_scan_step(*ins, st["state"], slots=st["slots"]), st["state"]
            y, last, saved = vmb.vmb_token_scan_fwd(*ins, initial_state=st["initial"], offsets=st["offsets"],
                                                    want_state=case["state"], want_saved=op == "scan_train")
            if op == "scan":
                return (y, last) if case["state"] else y
            d = vmb.vmb_token_scan_bwd(*ins, st["dy"], saved, offsets=st["offsets"])
            return (y, d["x"], d["delta"], d["A"], d["B"], d["C"], d["Dskip"], d["delta_bias"], d["z"])
        if op.startswith("norm"):
            y, total, scale, rstd = vmb.vmb_rms_norm_fwd(st["x"], st["weight"], st["residual"], eps=EPS, bits8=op == "norm8",
                                                         want_stats=op == "norm_train")
            if op != "norm_train":
                return y, total, scale
            d = vmb.vmb_rms_norm_bwd(st["x"] if total is None else total, st["weight"], rstd, st["dy"], dsum=st["dsum"])
            return y, total, d["x"], d["weight"]
        if op == "linear":
            return vmb.vmb_linear_fwd(st["x"], st["weight"], st["bias"], act=case["act"], residual=st["residual"])[0]
        if op == "linear8":
            return vmb.vmb_linear_fwd(st["x"], st["weight"], st["bias"], act=case["act"], residual=st["residual"],
                                      x_scale=st["x_scale"], weight_scale=st["weight_scale"])[0]
        d = vmb.vmb_linear_bwd(st["x"], st["weight"], st["dy"], st["pre"], act=case["act"], want_bias=case["bias"])
        return d["x"], d["weight"], d["bias"]
    if op.startswith("conv"):
        return _plain_conv_step(st, case) if op == "conv_step" else _plain_conv(st, case)
    if op.startswith("scan"):
        return _plain_scan_step(st, case) if op == "scan_step" else _plain_scan(st, case)
    if op.startswith("norm"):
        return _plain_norm(st, case)
    return _plain_linear(st, case)


# ------------------------------------------------------------------ the plain forms


def _activation(z, act):
    """act(z) and act'(z)."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def _places(st, case):
    """Of the tokens in order: each sequence's first and one past its last, the tokens' sequence and place in it."""
    x = st["x"]
    offsets = st["offsets"].long() if st["offsets"] is not None else torch.arange(case["B"] + 1, device=x.device) * case["T"]
    t = torch.arange(x.shape[0] * x.shape[1], device=x.device)
    seq = torch.searchsorted(offsets[1:].contiguous(), t, right=True)
    return offsets, seq, t - offsets[seq]


def _taps(st, case, seq, place):
    """fp32 [W, tokens, C]: the inputs that each token's taps see, zeros or the initial state before its sequence."""
    x, W = st["x"].reshape(-1, case["C"]).float(), case["W"]
    back = torch.arange(W - 1, -1, -1, device=x.device).view(-1, 1)
    at = torch.arange(x.shape[0], device=x.device) - back
    inside = (place - back >= 0).unsqueeze(-1)
    taps = torch.where(inside, x[at.clamp(min=0)], 0.0)
    if st["initial"] is not None:
        row = (W - 1 + place - back).clamp(0, W - 2) if W > 1 else None
        taps = torch.where(inside, taps, st["initial"].float()[seq.expand(W, -1), row])
    return taps


def _plain_conv(st, case):
    W, C, dt = case["W"], case["C"], st["x"].dtype
    if case["op"] == "conv_train":
        st = dict(st, initial=None)
    offsets, seq, place = _places(st, case)
    taps = _taps(st, case, seq, place)
    w = st["weight"].t().reshape(W, 1, C)
    y, slope = _activation((taps * w).sum(0) + st["bias"], case["act"])
    y = y.view(st["x"].shape).to(dt)
    if case["op"] == "conv":
        if not case["state"]:
            return y
        # the last W - 1 inputs of every sequence, of the initial state where it is shorter
        back = torch.arange(W - 1, 0, -1, device=y.device)
        at, n = offsets[1:, None] - back, (offsets[1:] - offsets[:-1]).unsqueeze(1)
        old = st["initial"].gather(1, (W - 1 + n - back).clamp(0, W - 2).unsqueeze(-1).expand(-1, -1, C))
        return y, torch.where((n >= back).unsqueeze(-1), st["x"].reshape(-1, C)[at.clamp(min=0)], old)
    g = st["dy"].reshape(-1, C).float() * slope
    ahead = torch.arange(W, device=y.device).view(-1, 1)  # token t's input meets the tap W - 1 - i of token t + i
    at, left = torch.arange(len(seq), device=y.device) + ahead, offsets[seq + 1]
    later = torch.where((at < left).unsqueeze(-1), g[at.clamp(max=len(seq) - 1)], 0.0)
    return y, (later * w.flip(0)).sum(0).view(st["x"].shape).to(dt), (taps * g).sum(1).t().contiguous(), g.sum(0)


def _plain_conv_step(st, case):
    B, W, T = case["B"], case["W"], case["T"]
    slots = torch.arange(B, device="cuda") if st["slots"] is None else st["slots"].long()
    used = slots >= 0
    row = torch.cat([st["state"][slots.clamp(min=0)], st["x"]], 1)
    seen = row.unfold(1, W, 1)[:, :T].float()  # [B, T, C, W]
    y = _activation((seen * st["weight"]).sum(-1) + st["bias"], case["act"])[0] * used.view(B, 1, 1)
    st["state"][slots[used]] = row[used, T:]
    return y.to(st["x"].dtype), st["state"]


def _running(a, b, longest):
    """h_t = a_t h_(t-1) + b_t along the first axis, by doubling: after step k a row joins the 2^k rows up to it."""
    k = 1
    while k < longest:
        b = torch.cat([b[:k], torch.addcmul(b[k:], a[k:], b[:-k])])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _plain_scan(st, case):
    """h_t = exp(delta A) h_(t-1) + delta x B, y = (C . h + D x) silu(z); a sequence's first token has no decay left, its
    initial state is in its input.  The adjoint runs the same way from the end."""
    D, N, dt, shape = case["D"], case["N"], st["x"].dtype, st["x"].shape
    offsets, seq, place = _places(st, case)
    x, raw, dtB, dtC = (st[n].reshape(-1, st[n].shape[-1]).float() for n in ("x", "delta", "Bm", "Cm"))
    raw = raw + st["bias"]
    delta, A = _softplus(raw), st["A"]
    a = torch.exp(delta.unsqueeze(-1) * A)
    first, longest = (place == 0).view(-1, 1, 1), int(case["T"])
    b = (delta * x).unsqueeze(-1) * dtB.unsqueeze(1)
    if st["initial"] is not None:
        b = torch.where(first, b + a * st["initial"][seq], b)
    h = _running(torch.where(first, 0.0, a), b, longest)
    out = (h * dtC.unsqueeze(1)).sum(-1) + st["D"] * x
    gate, slope = (1.0, None) if st["z"] is None else _activation(st["z"].reshape(-1, D).float(), "silu")
    y = (out * gate).view(shape).to(dt)
    if case["op"] == "scan":
        if not case["state"]:
            return y
        last = torch.where((offsets[1:] > offsets[:-1]).view(-1, 1, 1), h[(offsets[1:] - 1).clamp(min=0)],
                           st["initial"])
        return y, last
    dy = st["dy"].reshape(-1, D).float()
    g = dy * gate
    end = (place + 1 == (offsets[1:] - offsets[:-1])[seq]).view(-1, 1, 1)
    ahead = torch.where(end, 0.0, torch.cat([a[1:], a[:1]]))
    lam = _running(ahead.flip(0), (g.unsqueeze(-1) * dtC.unsqueeze(1)).flip(0), longest).flip(0)
    before = torch.where(first, 0.0, torch.cat([h[:1], h[:-1]]))
    decay = lam * before * a  # the gradient of delta A
    into = (lam * dtB.unsqueeze(1)).sum(-1)  # the gradient of delta x
    ddelta = ((decay * A).sum(-1) + into * x) / (1 + torch.exp(-raw))
    outs = [y, into * delta + g * st["D"], ddelta, (decay * delta.unsqueeze(-1)).sum(0),
            (lam * (delta * x).unsqueeze(-1)).sum(1), (h * g.unsqueeze(-1)).sum(1), (g * x).sum(0), ddelta.sum(0),
            None if slope is None else dy * out * slope]
    like = (y, st["x"], st["delta"], None, st["Bm"], st["Cm"], None, None, st["z"])
    return tuple(o if t is None else o.view(t.shape).to(dt) for o, t in zip(outs, like))


def _plain_scan_step(st, case):
    B, T, A = case["B"], case["T"], st["A"]
    slots = torch.arange(B, device="cuda") if st["slots"] is None else st["slots"].long()
    used = slots >= 0
    x, raw, dtB, dtC = (st[n].float().transpose(0, 1) for n in ("x", "delta", "Bm", "Cm"))
    delta = _softplus(raw + st["bias"])
    a = torch.exp(delta.unsqueeze(-1) * A)
    b = (delta * x).unsqueeze(-1) * dtB.unsqueeze(2)
    b[0] += a[0] * st["state"][slots.clamp(min=0)]
    h = _running(a, b, T)
    y = (h * dtC.unsqueeze(2)).sum(-1) + st["D"] * x
    if st["z"] is not None:
        y = y * _activation(st["z"].float().transpose(0, 1), "silu")[0]
    st["state"][slots[used]] = h[-1][used]
    return (y * used.view(1, B, 1)).transpose(0, 1).to(st["x"].dtype).contiguous(), st["state"]


def _plain_norm(st, case):
    dt, w = st["x"].dtype, st["weight"]
    total = None
    s = st["x"].float()
    if st["residual"] is not None:  # the residual stream is kept in its own type: that is what is normalised
        total = (s + st["residual"].float()).to(dt)
        s = total.float()
    rstd = torch.rsqrt(s.square().mean(1, keepdim=True) + EPS)
    n = s * rstd
    y = n * w
    if case["op"] == "norm":
        return y.to(dt), total, None
    if case["op"] == "norm8":
        scale = (y.abs().amax(1, keepdim=True) / 448).clamp(min=2.0 ** -100)
        return (y / scale).to(torch.float8_e4m3fn), total, scale.view(-1)
    dy = st["dy"].float()
    dn = dy * w
    dx = rstd * (dn - n * (dn * n).mean(1, keepdim=True)) + st["dsum"].float()
    return y.to(dt), total, dx.to(dt), (dy * n).sum(0)


def _plain_linear(st, case):
    x, w = st["x"].float(), st["weight"].float()
    if case["op"] == "linear_grad":
        d = st["dy"].float()
        if case["act"] != "none":
            d = d * _activation(st["pre"].float(), case["act"])[1]
        dt = st["x"].dtype
        return (d @ w).to(dt), (d.t() @ x).to(dt), d.sum(0) if case["bias"] else None
    y = x @ w.t()
    if case["op"] == "linear8":
        y = y * st["x_scale"].unsqueeze(1) * st["weight_scale"]
    if st["bias"] is not None:
        y = y + st["bias"]
    y = _activation(y, case["act"])[0]
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(torch.bfloat16)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    s, op = 4 if case["dtype"] == "f32" else 2, case["op"]
    if op.startswith("norm"):
        v, rows = case["rows"] * case["C"], case["rows"]
        more = 2 * v * s if case["residual"] else 0  # the residual in, the sum out
        if op == "norm":
            return {"bytes": 2 * s * v + more + 4 * case["C"], "flops": 5 * v}
        if op == "norm8":
            return {"bytes": (s + 1) * v + more + 4 * case["C"] + 4 * rows, "flops": 8 * v}
        return {"bytes": 5 * s * v + more + 8 * case["C"], "flops": 15 * v}
    if op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        e = 1 if op == "linear8" else 2
        if op == "linear_grad":
            return {"bytes": 2 * (2 * M * K + 2 * N * K + M * N * (1 if case["act"] == "none" else 2)) + 4 * N * case["bias"],
                    "flops": 4 * M * K * N}
        return {"bytes": e * (M * K + N * K) + 2 * M * N * (1 + case["residual"]) + 4 * N * case["bias"]
                + (4 * (M + N) if e == 1 else 0), "flops": 2 * M * K * N}
    lens = _ints(case.get("lens", ""))
    tokens = sum(lens) if lens else case["B"] * case["T"]
    if op.startswith("conv"):
        C, W = case["C"], case["W"]
        v, params = tokens * C, 4 * C * (W + 1)
        act = 4 if case["act"] == "silu" else 0
        if op == "conv_step":
            rows = case["B"] - (case["B"] // 16 if case["pool"] else 0)
            return {"bytes": 2 * s * v + 2 * s * rows * (W - 1) * C + params, "flops": (2 * W + act) * v}
        if op == "conv":
            return {"bytes": 2 * s * v + (2 * s * case["B"] * (W - 1) * C if case["state"] else 0) + params, "flops": (2 * W + act) * v}
        return {"bytes": 4 * s * v + 2 * params, "flops": (8 * W + 3 * act) * v}
    D, N = case["D"], case["N"]
    v, bc, gate = tokens * D, 2 * tokens * N, 1 if case["gate"] else 0
    # a state of a channel and token: delta A, its exponential, its input, the recurrence, C . h
    flops = v * (7 * N + 8 + 5 * gate)
    if op == "scan_step":
        rows = case["B"] - (case["B"] // 16 if case["pool"] else 0)
        return {"bytes": s * (v * (3 + gate) + bc) + 8 * rows * D * N + 4 * D * (N + 2), "flops": flops}
    if op == "scan":
        return {"bytes": s * (v * (3 + gate) + bc) + (8 * case["B"] * D * N if case["state"] else 0) + 4 * D * (N + 2), "flops": flops}
    # the gradients read the inputs and dy, write one gradient for each input, and take the recurrence's reverse
    return {"bytes": s * (v * (6 + 2 * gate) + 2 * bc) + 8 * D * (N + 2), "flops": flops + v * (15 * N + 20 + 8 * gate)}


# ------------------------------------------------------------------ the definitions in 64 bits


def _spans(st, case):
    """(batch row, first token, one past the last) of every sequence."""
    if st["offsets"] is None:
        return [(b, 0, case["T"]) for b in range(case["B"])]
    at = st["offsets"].tolist()
    return [(0, at[i], at[i + 1]) for i in range(len(at) - 1)]


def _act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(st, case)
    if case["op"].startswith("linear"):
        return _exact_linear(st, case)
    if case["op"].startswith("conv"):
        return _exact_conv(st, case)
    return _exact_scan(st, case)


def _conv64(x, first, w, bias, act):
    """One sequence [n, C] behind its W - 1 earlier inputs, tap by tap."""
    full, n = torch.cat([first, x]), x.shape[0]
    z = bias.expand(n, -1)
    for j in range(w.shape[1]):
        z = z + full[j:j + n] * w[:, j]
    return _act64(z, act)


def _exact_conv(st, case):
    W, C, op = case["W"], case["C"], case["op"]
    w, bias, x = st["weight"].double().requires_grad_(), st["bias"].double().requires_grad_(), st["x"].double()
    if op == "conv_step":
        slots = list(range(case["B"])) if st["slots"] is None else st["slots"].tolist()
        state, y = st["state"].double(), torch.zeros_like(x)
        with torch.no_grad():
            for b, slot in enumerate(slots):
                if slot >= 0:
                    y[b] = _conv64(x[b], state[slot], w, bias, case["act"])
                    state[slot] = torch.cat([state[slot], x[b]])[x.shape[1]:]
        return y, state
    y, last = torch.zeros_like(x), []
    train = op == "conv_train"
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(bias)
    with torch.set_grad_enabled(train):
        for i, (b, t0, t1) in enumerate(_spans(st, case)):
            first = x.new_zeros(W - 1, C) if train or st["initial"] is None else st["initial"][i].double()
            xs = x[b, t0:t1].clone().requires_grad_(train)
            out = _conv64(xs, first, w, bias, case["act"])
            y[b, t0:t1] = out.detach()
            last.append(torch.cat([first, xs.detach()])[t1 - t0:])
            if train and t1 > t0:
                g = torch.autograd.grad(out, (xs, w, bias), st["dy"][b, t0:t1].double())
                dx[b, t0:t1] = g[0]
                dw, db = dw + g[1], db + g[2]
    if train:
        return y, dx, dw.detach(), db.detach()
    return (y, torch.stack(last)) if case["state"] else y


def _exact_scan(st, case):
    """Token after token over all sequences at once, each padded to the longest; gradients by automatic differentiation in
    stretches of 64 tokens."""
    D, N, op = case["D"], case["N"], case["op"]
    A, skip, bias = (st[n].double() for n in ("A", "D", "bias"))
    if op == "scan_step":
        B = case["B"]
        slots = list(range(B)) if st["slots"] is None else st["slots"].tolist()
        spans, rows = [(b, 0, case["T"]) for b in range(B)], [b for b in range(B) if slots[b] >= 0]
    else:
        spans = _spans(st, case)
        rows = list(range(len(spans)))
    most = max(t1 - t0 for _, t0, t1 in spans)
    if most * len(spans) * D * N > (6e9 if op == "scan" else 2.5e9) * 4:
        return None
    names = ["x", "delta", "Bm", "Cm"] + (["z"] if st["z"] is not None else []) + (["dy"] if op == "scan_train" else [])
    at = {}
    for n in names:
        p = torch.zeros(most, len(spans), st[n].shape[-1], dtype=torch.float64, device="cuda")
        for i, (b, t0, t1) in enumerate(spans):
            p[:t1 - t0, i] = st[n][b, t0:t1]
        at[n] = p
    alive = torch.tensor([[t < t1 - t0 for _, t0, t1 in spans] for t in range(most)], device="cuda").view(most, -1, 1, 1)

    def token(h, t, x, raw, dtB, dtC, z, A, skip, bias):
        delta = torch.logaddexp(raw + bias, torch.zeros((), dtype=torch.float64, device="cuda"))
        new = torch.exp(delta.unsqueeze(-1) * A) * h + torch.einsum("bd,bn->bdn", delta * x, dtB)
        h = torch.where(alive[t], new, h)
        y = torch.einsum("bdn,bn->bd", h, dtC) + skip * x
        return h, y if z is None else y * z * torch.sigmoid(z)

    def ins(t):
        return [at[n][t] if n in at else None for n in ("x", "delta", "Bm", "Cm", "z")]

    def back(p):
        out = torch.zeros(st["x"].shape[:2] + p.shape[2:], dtype=torch.float64, device="cuda")
        for i, (b, t0, t1) in enumerate(spans):
            out[b, t0:t1] = p[:t1 - t0, i]
        return out

    h = torch.zeros(len(spans), D, N, dtype=torch.float64, device="cuda")
    if op == "scan_step":
        state = st["state"].double()
        h[rows] = state[[slots[b] for b in rows]]
    elif st["initial"] is not None:
        h = st["initial"].double()
    y, kept = torch.empty_like(at["x"]), []
    for t in range(most):
        if t % 64 == 0:
            kept.append(h)
        h, y[t] = token(h, t, *ins(t), A, skip, bias)
    if op == "scan_step":
        y = back(y)
        for b in range(len(spans)):
            if b in rows:
                state[slots[b]] = h[b]
            else:
                y[b] = 0
        return y, state
    if op == "scan":
        return (back(y), h) if case["state"] else back(y)
    weights = [v.requires_grad_() for v in (A, skip, bias)]
    total = [torch.zeros_like(v) for v in weights]
    grads = {n: torch.zeros_like(at[n]) for n in names if n != "dy"}
    dh = torch.zeros_like(h)
    for j in range(len(kept) - 1, -1, -1):
        h0 = kept[j].detach().requires_grad_()
        h, got, leaves = h0, 0.0, []
        for t in range(64 * j, min(most, 64 * j + 64)):
            these = [None if v is None else v.clone().requires_grad_() for v in ins(t)]
            leaves.append(these)
            h, out = token(h, t, *these, *weights)
            got = got + (out * at["dy"][t]).sum()
        got = got + (h * dh).sum()
        flat = [v for these in leaves for v in these if v is not None]
        d = torch.autograd.grad(got, [h0, *weights, *flat])
        dh, total = d[0], [a + b for a, b in zip(total, d[1:4])]
        d = list(d[4:])
        for t in range(64 * j, min(most, 64 * j + 64)):
            for n in grads:
                grads[n][t] = d.pop(0)
    return (back(y), back(grads["x"]), back(grads["delta"]), total[0], back(grads["Bm"]), back(grads["Cm"]), total[1], total[2],
            back(grads["z"]) if "z" in grads else None)


def _exact_norm(st, case):
    s, total = st["x"].double(), None
    if st["residual"] is not None:
        total = st["x"] + st["residual"]  # rounded to the stream's type by definition
        s = total.double()
    w = st["weight"].double()
    length = torch.linalg.vector_norm(s, dim=1, keepdim=True)
    r = 1 / torch.sqrt(length * length / case["C"] + EPS)
    y = s * w * r
    if case["op"] == "norm":
        return y, total, None
    if case["op"] == "norm8":
        scale = (y.abs().max(1).values / 448).clamp(min=2.0 ** -100)
        return y / scale.unsqueeze(1), total, scale
    dy = st["dy"].double()
    dx = dy * w * r - s * r ** 3 / case["C"] * (dy * w * s).sum(1, keepdim=True) + st["dsum"].double()
    return y, total, dx, torch.einsum("rc,rc,rx->c", dy, s, r)


def _exact_linear(st, case):
    x, w = st["x"].double(), st["weight"].double()
    if case["op"] == "linear_grad":
        d = st["dy"].double()
        if case["act"] != "none":
            p = st["pre"].double().requires_grad_()
            d, = torch.autograd.grad(_act64(p, case["act"]), p, d)
        return torch.einsum("mn,nk->mk", d, w), torch.einsum("mn,mk->nk", d, x), d.sum(0) if case["bias"] else None
    if case["op"] == "linear8":
        x, w = x * st["x_scale"].double().unsqueeze(1), w * st["weight_scale"].double().unsqueeze(1)
    y = torch.einsum("mk,nk->mn", x, w)
    if st["bias"] is not None:
        y += st["bias"].double()
    y = _act64(y, case["act"])
    return y if st["residual"] is None else y + st["residual"].double()
