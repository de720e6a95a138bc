"""The gated delta rule on the GPU against the recurrence in 64 bits.

Tolerances (2-norm of the difference over that of the reference, of every output):
  fp32: operands carry 22 bits and sums 24; a value passes at most about eight products of up to 128 terms between
    roundings, so a relative error of 16 * 2^-22 = 4e-6 is expected at the worst, 2e-5 allowed.
  bf16 outputs: their own rounding is 2^-9 / sqrt(3) = 1.1e-3 (up to 2e-3 over a mantissa); gradients pass up to four
    more roundings of operands to bf16: sqrt(5) * 2e-3 = 4.5e-3, 1e-2 allowed.  fp32 states of bf16 inputs: operands
    of 16 bits, 2^-17 each, about eight of them: 6e-5 at the worst in sum, 2e-5 in quadrature, 4e-5 allowed."""
import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def tol(dtype, state=False):
    return 2e-5 if dtype == torch.float32 else 4e-5 if state else 1e-2


def close(got, want, limit, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    off, size = (got - want).norm().item(), want.norm().item()
    assert off <= limit * size or off <= 1e-12, f"{what}: {off / max(size, 1e-300):.2e} > {limit:.0e}"


def gpu(xs):
    return [x.cuda() for x in xs]


SIZES = [  # B, T, Hk, Hv, Dk, Dv
    (1, 1, 1, 1, 64, 64), (2, 2, 1, 2, 9, 5), (1, 15, 1, 1, 16, 16), (2, 63, 2, 2, 64, 64), (1, 64, 1, 3, 64, 64),
    (3, 65, 2, 2, 48, 80), (1, 129, 1, 1, 128, 128), (2, 130, 2, 4, 127, 33), (1, 200, 1, 2, 100, 130), (2, 190, 3, 3, 1, 1),
    (1, 700, 1, 1, 64, 64), (1, 520, 1, 2, 128, 72), (40, 70, 2, 4, 32, 64),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_gradients(size, dtype):
    import paper_2412_16602_gb300 as vmb
    dt = TYPES[dtype]
    B, T, Hk, Hv, Dk, Dv = size
    x = ref.inputs(*size, seed=sum(size), dtype=dt)
    gen = torch.Generator().manual_seed(7)
    init, dfinal = torch.randn(B, Hv, Dk, Dv, generator=gen) * 0.3, torch.randn(B, Hv, Dk, Dv, generator=gen)
    do = torch.randn(B, T, Hv, Dv, generator=gen).to(dt)
    o, S, _ = ref.forward(*x, init)
    d = ref.backward(*x, do, init, dfinal)
    c = gpu(x)
    go, gS, saved = vmb.vmb_delta_rule_fwd(*c, initial_state=init.cuda(), want_state=True, want_saved=True)
    gd = vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved, dfinal_state=dfinal.cuda(), want_initial=True)
    close(go, o, tol(dt), "o")
    close(gS, S, tol(dt, True), "final state")
    for n in ("q", "k", "v", "g", "beta"):
        close(gd[n], d[n], tol(dt) * (3 if n == "g" else 1), n)  # dg is a difference of such sums
    close(gd["initial_state"], d["initial_state"], tol(dt, True), "initial state")
    # without a final state or kept states: the same outputs
    assert torch.equal(vmb.vmb_delta_rule_fwd(*c, initial_state=init.cuda())[0], go)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_initial_state(dtype):
    import paper_2412_16602_gb300 as vmb
    x = ref.inputs(2, 100, 1, 2, 64, 64, 5, TYPES[dtype])
    do = torch.randn(2, 100, 2, 64, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype])
    c = gpu(x)
    o, S, saved = vmb.vmb_delta_rule_fwd(*c, want_saved=True)
    assert S is None
    close(o, ref.forward(*x)[0], tol(TYPES[dtype]), "o")
    d, gd = ref.backward(*x, do), vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved)
    assert "initial_state" not in gd
    for n in ("q", "k", "v", "g", "beta"):
        close(gd[n], d[n], tol(TYPES[dtype]) * (3 if n == "g" else 1), n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [(1, 64, 0, 130, 65), (0, 0, 3), (700,), (5, 0), (64, 64, 64, 1)])
def test_packed_sequences(lens, dtype):
    """Every sequence is as if alone; empty ones pass their state on."""
    import paper_2412_16602_gb300 as vmb
    dt, total, Hk, Hv, Dk, Dv = TYPES[dtype], sum(lens), 1, 2, 64, 48
    x = ref.inputs(1, total, Hk, Hv, Dk, Dv, 11, dt)
    gen = torch.Generator().manual_seed(2)
    init, dfinal = (torch.randn(len(lens), Hv, Dk, Dv, generator=gen) for _ in range(2))
    do = torch.randn(1, total, Hv, Dv, generator=gen).to(dt)
    offsets = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32).cuda()
    kw = dict(offsets=offsets, max_len=max(lens))
    c = gpu(x)
    o, S, saved = vmb.vmb_delta_rule_fwd(*c, initial_state=init.cuda(), want_state=True, want_saved=True, **kw)
    gd = vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved, dfinal_state=dfinal.cuda(), want_initial=True, **kw)
    assert vmb.vmb_read_status(vmb.delta_workspace()) == vmb.VMB_OK
    at = 0
    for i, n in enumerate(lens):
        part = [t[:, at:at + n] for t in x]
        wo, wS, _ = ref.forward(*part, init[i:i + 1])
        wd = ref.backward(*part, do[:, at:at + n], init[i:i + 1], dfinal[i:i + 1])
        close(S[i:i + 1], wS, tol(dt, True), f"state {i}")
        close(gd["initial_state"][i:i + 1], wd["initial_state"], tol(dt, True), f"initial {i}")
        if n:
            close(o[:, at:at + n], wo, tol(dt), f"o {i}")
            for name in ("q", "k", "v", "g", "beta"):
                close(gd[name][:, at:at + n], wd[name], tol(dt) * (3 if name == "g" else 1), f"{name} {i}")
        at += n


def test_offsets_out_of_range_are_reported():
    import paper_2412_16602_gb300 as vmb
    x = gpu(ref.inputs(1, 20, 1, 1, 16, 16, 3))
    for bad in ([0, 10, 40], [0, 12, 8], [-3, 5, 20], [0, 20, 20]):
        ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
        longest = 12 if bad == [0, 20, 20] else 20
        o, _, _ = vmb.vmb_delta_rule_fwd(*x, offsets=torch.tensor(bad, dtype=torch.int32).cuda(), max_len=longest, workspace=ws,
                                         o=torch.zeros(1, 20, 1, 16, device="cuda"))
        assert vmb.vmb_read_status(ws) == vmb.VMB_ERR_BOUNDS
        assert vmb.vmb_read_status(ws) == vmb.VMB_OK  # cleared
        assert torch.isfinite(o).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 70, 600])
def test_strided_rows_and_odd_addresses(T, dtype):
    """q, k, v as parts of one projection's row, and every tensor one element past its alignment."""
    import paper_2412_16602_gb300 as vmb
    dt = TYPES[dtype]
    torch.manual_seed(9)
    q, k, v, g, beta = gpu(ref.inputs(2, T, 2, 2, 64, 32, 13, dt))
    do = torch.randn(2, T, 2, 32, device="cuda").to(dt)
    want, S, saved = vmb.vmb_delta_rule_fwd(q, k, v, g, beta, want_state=True, want_saved=True)
    dwant = vmb.vmb_delta_rule_bwd(q, k, v, g, beta, do, saved)
    for pad in (0, 8, 1):
        row = torch.cat([t.reshape(2, T, -1) for t in (q, k, v)] + [torch.zeros(2, T, pad, dtype=dt, device="cuda")], -1)
        cut = [row[..., :128].view(2, T, 2, 64), row[..., 128:256].view(2, T, 2, 64), row[..., 256:320].view(2, T, 2, 32)] \
            if T > 1 else [row[..., a:b].unflatten(-1, (2, d)) for a, b, d in ((0, 128, 64), (128, 256, 64), (256, 320, 32))]
        o, S2, saved = vmb.vmb_delta_rule_fwd(*cut, g, beta, want_state=True, want_saved=True)
        assert torch.equal(o, want) and torch.equal(S, S2)
        d = vmb.vmb_delta_rule_bwd(*cut, g, beta, do, saved)
        assert all(torch.equal(d[n], dwant[n]) for n in dwant)

    def off(t):
        b = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        b[1:] = t.reshape(-1)
        return b[1:].view(t.shape)

    odd = [off(t) for t in (q, k, v, g, beta)]
    o, S2, saved = vmb.vmb_delta_rule_fwd(*odd, want_state=True, want_saved=True, o=off(want))
    assert torch.equal(o, want) and torch.equal(S, S2)
    d = vmb.vmb_delta_rule_bwd(*odd, off(do), saved)
    assert all(torch.equal(d[n], dwant[n]) for n in dwant)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_resets_and_masked_tokens(dtype):
    """g = -inf (and the type's lowest value) forgets everything before; beta = 0 leaves the state to its decay."""
    import paper_2412_16602_gb300 as vmb
    dt = TYPES[dtype]
    q, k, v, g, beta = ref.inputs(1, 150, 1, 2, 64, 64, 17, dt)
    g[:, 40], g[:, 64], g[:, 100:110, 0], g[:, 120, 1] = -float("inf"), torch.finfo(dt).min, -float("inf"), -90.0
    beta[:, 20:30], beta[:, 66] = 0, 0
    do = torch.randn(1, 150, 2, 64, generator=torch.Generator().manual_seed(4)).to(dt)
    init = torch.randn(1, 2, 64, 64, generator=torch.Generator().manual_seed(5))
    o, S, _ = ref.forward(q, k, v, g, beta, init)
    d = ref.backward(q, k, v, g, beta, do, init)
    c = gpu([q, k, v, g, beta])
    go, gS, saved = vmb.vmb_delta_rule_fwd(*c, initial_state=init.cuda(), want_state=True, want_saved=True)
    gd = vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved, want_initial=True)
    close(go, o, tol(dt), "o")
    close(gS, S, tol(dt, True), "state")
    for n in ("q", "k", "v", "beta"):
        close(gd[n], d[n], tol(dt), n)
    close(gd["g"], d["g"], tol(dt) * 3, "g")
    close(gd["initial_state"], d["initial_state"], tol(dt, True), "initial state")  # through the tokens before the reset
    alone = vmb.vmb_delta_rule_fwd(*[t[:, 40:] for t in c])[0]  # nothing crosses the reset
    close(go[:, 40:], alone.double().cpu(), tol(dt), "after the reset")
    close(vmb.vmb_delta_rule_fwd(*c, initial_state=5 * init.cuda())[0][:, 40:], o[:, 40:], tol(dt), "whatever was before")


def test_what_is_not_a_number_stays_in_its_head():
    """... and channel, and reaches the tokens after it and the others of its block of 16."""
    import paper_2412_16602_gb300 as vmb
    c = gpu(ref.inputs(2, 90, 2, 2, 64, 64, 19))
    want = vmb.vmb_delta_rule_fwd(*c)[0]
    c[2][1, 30, 0, 5] = float("nan")
    o = vmb.vmb_delta_rule_fwd(*c)[0]
    assert torch.equal(o[0], want[0]) and torch.equal(o[1, :, 1], want[1, :, 1])
    assert torch.equal(o[1, :16, 0], want[1, :16, 0]) and torch.isnan(o[1, 30:, 0, 5]).all()


def test_long_memory():
    """No decay at all over many chunks and segments: the state keeps its digits."""
    import paper_2412_16602_gb300 as vmb
    q, k, v, g, beta = ref.inputs(1, 2000, 1, 1, 64, 64, 23)
    g.zero_()
    o, S, _ = ref.forward(q, k, v, g, beta)
    c = gpu([q, k, v, g, beta])
    go, gS, _ = vmb.vmb_delta_rule_fwd(*c, want_state=True)
    close(go, o, 2e-5, "o")
    close(gS, S, 2e-5, "state")


def test_gradients_against_differences():
    """Central differences of the GPU's own forward in fp32: the slope along a random direction, step h.  Its error is
    the forward's rounding over h (1e-6 |L| / h) and the third derivative's h^2 / 6; 2e-3 of the slope's size allowed."""
    import paper_2412_16602_gb300 as vmb
    x = ref.inputs(2, 80, 1, 2, 64, 64, 29)
    gen = torch.Generator().manual_seed(6)
    do = torch.randn(2, 80, 2, 64, generator=gen)
    c = gpu(x)
    _, _, saved = vmb.vmb_delta_rule_fwd(*c, want_saved=True)
    d = vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved)
    for i, n in enumerate(("q", "k", "v", "g", "beta")):
        step = torch.randn(x[i].shape, generator=gen)
        step = step * (x[i].norm() / step.norm())
        h = 1e-2
        values = []
        for s in (h, -h):
            y = [(t + s * step if j == i else t).cuda() for j, t in enumerate(x)]
            values.append((vmb.vmb_delta_rule_fwd(*y)[0].double().cpu() * do.double()).sum().item())
        slope, want = (values[0] - values[1]) / (2 * h), (d[n].double().cpu() * step.double()).sum().item()
        size = d[n].double().norm().item() * step.double().norm().item() / step.numel() ** 0.5
        assert abs(slope - want) <= 2e-3 * max(abs(want), size) + 1e-3 * size, (n, slope, want)


def test_deterministic_on_another_stream():
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(10)
    c = gpu(ref.inputs(1, 900, 1, 2, 64, 64, 31, torch.bfloat16))
    do = torch.randn(1, 900, 2, 64, device="cuda").bfloat16()
    o, _, saved = vmb.vmb_delta_rule_fwd(*c, want_saved=True)
    d = vmb.vmb_delta_rule_bwd(*c, do, saved)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            o2, _, saved2 = vmb.vmb_delta_rule_fwd(*c, want_saved=True, workspace=ws)
            d2 = vmb.vmb_delta_rule_bwd(*c, do, saved2, workspace=ws)
    s.synchronize()
    assert torch.equal(o, o2) and all(torch.equal(d[n], d2[n]) for n in d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 6, 6, 64, 64), (5, 1, 2, 4, 128, 128), (3, 4, 1, 3, 48, 80), (2, 2, 1, 1, 1, 1),
                                  (2, 3, 1, 2, 127, 131), (40, 1, 2, 2, 65, 64)])
def test_step(size, dtype):
    import paper_2412_16602_gb300 as vmb
    dt = TYPES[dtype]
    B, T, Hk, Hv, Dk, Dv = size
    x = ref.inputs(*size, seed=37, dtype=dt)
    init = torch.randn(B, Hv, Dk, Dv, generator=torch.Generator().manual_seed(8))
    o, S, _ = ref.forward(*x, init)
    state = init.cuda()
    go = vmb.vmb_delta_rule_step(*gpu(x), state)
    close(go, o, tol(dt), "o")
    close(state, S, 2e-6, "state")  # fp32 arithmetic throughout, at most 128 terms
    # the same through slots of a pool, with padding
    pool = torch.full((B + 3, Hv, Dk, Dv), 7.0, device="cuda")
    slots = torch.randperm(B + 3)[:B].to(torch.int32)
    pool[slots.long().cuda()] = init.cuda()
    slots[B // 2] = -1 if B > 1 else slots[B // 2]
    before = pool.clone()
    go2 = vmb.vmb_delta_rule_step(*gpu(x), pool, slots=slots.cuda())
    for b in range(B):
        if slots[b] < 0:
            assert go2[b].abs().max().item() == 0
        else:
            assert torch.equal(go2[b], go[b]) and torch.equal(pool[slots[b]], state[b])
    idle = [i for i in range(B + 3) if i not in slots.tolist()]
    assert torch.equal(pool[idle], before[idle])
    # a slot behind the pool is left out as well
    assert vmb.vmb_delta_rule_step(*gpu(x), pool, slots=torch.full((B,), B + 3, dtype=torch.int32, device="cuda")).abs().max().item() == 0


def test_prefill_then_steps():
    """The chunked form's final state goes on token by token as the whole sequence would."""
    import paper_2412_16602_gb300 as vmb
    c = gpu(ref.inputs(2, 100, 1, 2, 64, 64, 41))
    whole, final, _ = vmb.vmb_delta_rule_fwd(*c, want_state=True)
    o, state, _ = vmb.vmb_delta_rule_fwd(*[t[:, :90].contiguous() for t in c], want_state=True)
    close(o, whole[:, :90].double().cpu(), 2e-5)
    for t in range(90, 100):
        close(vmb.vmb_delta_rule_step(*[x[:, t:t + 1] for x in c[:3]], *[x[:, t:t + 1].contiguous() for x in c[3:]], state),
              whole[:, t:t + 1].double().cpu(), 2e-5)
    close(state, final.double().cpu(), 2e-5)


def test_empty_problems():
    import paper_2412_16602_gb300 as vmb
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    init = torch.randn(2, 1, 8, 8, device="cuda")
    o, S, saved = vmb.vmb_delta_rule_fwd(z(2, 0, 1, 8), z(2, 0, 1, 8), z(2, 0, 1, 8), z(2, 0, 1), z(2, 0, 1), initial_state=init,
                                         want_state=True, want_saved=True)
    assert o.shape == (2, 0, 1, 8) and torch.equal(S, init)
    d = vmb.vmb_delta_rule_bwd(z(2, 0, 1, 8), z(2, 0, 1, 8), z(2, 0, 1, 8), z(2, 0, 1), z(2, 0, 1), z(2, 0, 1, 8), saved,
                               dfinal_state=init, want_initial=True)
    assert torch.equal(d["initial_state"], init)
    vmb.vmb_delta_rule_fwd(z(0, 5, 1, 8), z(0, 5, 1, 8), z(0, 5, 1, 8), z(0, 5, 1), z(0, 5, 1))
    vmb.vmb_delta_rule_step(z(0, 1, 1, 8), z(0, 1, 1, 8), z(0, 1, 1, 8), z(0, 1, 1), z(0, 1, 1), z(3, 1, 8, 8))


def test_refusals():
    import paper_2412_16602_gb300 as vmb
    q, k, v, g, beta = gpu(ref.inputs(1, 8, 2, 2, 16, 16, 43))
    fwd = vmb.vmb_delta_rule_fwd
    for bad in ([q.cpu(), k, v, g, beta], [q, k[:, :4], v, g, beta], [q, k, v, g[..., :1], beta], [q, k, v, g, beta.bfloat16()],
                [q, k, v[:, :, :1], g[..., :1].contiguous(), beta[..., :1].contiguous()], [q.transpose(2, 3), k, v, g, beta]):
        with pytest.raises((ValueError, TypeError)):
            fwd(*bad)
    with pytest.raises(TypeError):
        fwd(*[t.half() for t in (q, k, v, g, beta)])
    with pytest.raises(ValueError):
        fwd(q, k, v, g, beta, initial_state=torch.zeros(1, 2, 16, 8, device="cuda"))
    with pytest.raises(ValueError):
        fwd(q, k, v, g, beta, offsets=torch.tensor([0, 8], dtype=torch.int32).cuda())  # max_len is missing
    with pytest.raises(ValueError):
        fwd(q, k, v, g, beta, offsets=torch.tensor([0, 8]).cuda(), max_len=8)  # int64
    with pytest.raises(vmb.VmbError) as e:
        fwd(*gpu(ref.inputs(1, 8, 1, 1, 129, 16, 43)))
    assert e.value.status == vmb.VMB_ERR_UNSUPPORTED
    with pytest.raises(vmb.VmbError) as e:
        fwd(q, k, v, g, beta, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == vmb.VMB_ERR_WORKSPACE
    with pytest.raises(ValueError):
        vmb.vmb_delta_rule_bwd(q, k, v, g, beta, v, torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(vmb.VmbError) as e:
        vmb.vmb_delta_rule_step(q, k, v, g, beta, torch.zeros(0, 2, 16, 16, device="cuda"))
    assert e.value.status == vmb.VMB_ERR_INVALID_ARG
