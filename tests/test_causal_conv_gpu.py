"""The short causal convolution against its definition in 64 bits: dense and packed sequences, states, gradients, steps.

Tolerances: z sums W products and the bias, 5 roundings of 2^-24 relative to the terms' magnitudes, which in the norm of a
whole tensor exceed |z| by at most 4 here; SiLU adds an exponential and a reciprocal of about 2^-22 each.  So 2^-19 covers
fp32; bf16 storage adds one rounding of at most 2^-8.  Sums over the tokens of weights' gradients have a condition of up to
sqrt(tokens) for terms of random sign, below 2^5 here."""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
OUT = {F32: 2.0 ** -19, BF16: 2.0 ** -8 + 2.0 ** -19}
SUM = 2.0 ** -14


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    return vmb


def make(seed, B, T, C, W, dtype, half=False, bias=True, n=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x = r(B, T, 2 * C).to(dtype)[..., C:] if half else r(B, T, C).to(dtype)
    n = B if n is None else n
    return x, 0.5 * r(C, W), r(C) if bias else None, r(n, W - 1, C).to(dtype), r(B, T, C).to(dtype), r(n, W - 1, C).to(dtype)


def d(t):
    return None if t is None else t.double().cpu()


CASES = [(2, 37, 24, 4, "silu", F32, False), (1, 1, 8, 4, "silu", BF16, False), (3, 5, 7, 3, "none", F32, True), (2, 130, 96, 2, "silu", BF16, True),
         (1, 300, 264, 1, "silu", F32, False), (2, 2, 40, 4, "none", BF16, False), (1, 67, 1032, 4, "silu", BF16, False), (4, 0, 16, 4, "silu", F32, False),
         (2, 33, 13, 4, "silu", BF16, True), (1, 17, 2056, 3, "silu", F32, False)]
PACKED = [(3, [0, 1, 2, 3, 50, 0, 17, 64], 5), (0, [1], 0), (0, [40, 0, 0, 33], 0), (7, [0, 0], 9), (0, [16, 16, 16], 16)]


@pytest.mark.parametrize("B,T,C,W,act,dtype,half", CASES)
@pytest.mark.parametrize("state", [False, True])
def test_forward_and_gradients(vmb, B, T, C, W, act, dtype, half, state):
    x, w, b, init, dy, dlast = make(1, B, T, C, W, dtype, half)
    init, dlast = (init, dlast) if state else (None, None)
    y, last = vmb.vmb_causal_conv_fwd(x, w, b, act=act, initial_state=init, want_state=state)
    yr, lr = ref.conv(d(x), d(w), d(b), d(init), act=act)
    assert ref.rel(y, yr) <= OUT[dtype]
    if state:
        assert torch.equal(last.cpu(), lr.to(dtype))
    got = vmb.vmb_causal_conv_bwd(x, w, b, dy, act=act, initial_state=init, dfinal_state=dlast, want_initial=state)
    want = ref.gradients(lambda x, w, b, i: ref.conv(x, w, b, i, act=act), (x, w, b, init), (dy, dlast))
    assert ref.rel(got["x"], want[0]) <= OUT[dtype]
    if T:
        assert ref.rel(got["weight"], want[1]) <= SUM and ref.rel(got["bias"], want[2]) <= SUM
    else:
        assert not got["weight"].any() and not got["bias"].any()
    if state:
        assert ref.rel(got["initial_state"], want[3]) <= OUT[dtype]


@pytest.mark.parametrize("lead,lens,tail", PACKED)
@pytest.mark.parametrize("C,W,dtype", [(24, 4, F32), (40, 3, BF16), (5, 4, BF16), (8, 2, F32)])
def test_packed(vmb, lead, lens, tail, C, W, dtype):
    at = [lead]
    for n in lens:
        at.append(at[-1] + n)
    T = at[-1] + tail
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    x, w, b, init, dy, dlast = make(2, 1, T, C, W, dtype, n=len(lens))
    y, last = vmb.vmb_causal_conv_fwd(x, w, b, initial_state=init, offsets=offsets, want_state=True, y=torch.full_like(x, 7.0))
    yr, lr = ref.conv(d(x), d(w), d(b), d(init), offsets)
    assert ref.rel(y, yr) <= OUT[dtype] and torch.equal(last.cpu(), lr.to(dtype))
    assert not y[:, :lead].any() and not y[:, at[-1]:].any()
    got = vmb.vmb_causal_conv_bwd(x, w, b, dy, initial_state=init, dfinal_state=dlast, offsets=offsets, want_initial=True)
    want = ref.gradients(lambda x, w, b, i: ref.conv(x, w, b, i, offsets), (x, w, b, init), (dy, dlast))
    assert ref.rel(got["x"], want[0]) <= OUT[dtype] and ref.rel(got["initial_state"], want[3]) <= OUT[dtype]
    assert ref.rel(got["weight"], want[1]) <= SUM and ref.rel(got["bias"], want[2]) <= SUM
    assert not got["x"][:, :lead].any() and not got["x"][:, at[-1]:].any()


@pytest.mark.parametrize("B,T,C,W,dtype,slots", [(5, 1, 40, 4, BF16, True), (3, 3, 7, 3, F32, True), (4, 2, 264, 2, F32, False), (2, 1, 16, 1, BF16, False),
                                                 (1, 6, 1040, 4, BF16, True)])
def test_steps(vmb, B, T, C, W, dtype, slots):
    x, w, b, _, _, _ = make(3, B, T, C, W, dtype)
    pool = torch.randn(B + 4, W - 1, C, device="cuda").to(dtype)
    old, at = pool.clone(), torch.arange(B, dtype=torch.int32)
    if slots:
        at = torch.randperm(B + 4, generator=torch.Generator().manual_seed(1))[:B].to(torch.int32)
        if B > 1:
            at[1] = -1
    y = vmb.vmb_causal_conv_step(x, w, b, pool, slots=at.cuda() if slots else None)
    used = [i for i in range(B) if at[i] >= 0]
    yr, lr = ref.conv(d(x[used]), d(w), d(b), d(old[at[used].long()]))
    assert ref.rel(y[used], yr) <= OUT[dtype]
    want = old.clone()
    want[at[used].long()] = lr.to(dtype).cuda()
    assert torch.equal(pool, want)
    assert not y[[i for i in range(B) if at[i] < 0]].any()


def test_steps_continue_a_prompt(vmb):
    x, w, b, _, _, _ = make(4, 2, 41, 48, 4, F32)
    whole, _ = vmb.vmb_causal_conv_fwd(x, w, b)
    head, state = vmb.vmb_causal_conv_fwd(x[:, :38], w, b, want_state=True)  # (a strided view)
    tail = [vmb.vmb_causal_conv_step(x[:, t:t + 1], w, b, state) for t in range(38, 41)]
    assert torch.equal(torch.cat([head, *tail], 1), whole)


def test_no_bias(vmb):
    x, w, _, _, dy, _ = make(5, 2, 20, 16, 4, F32, bias=False)
    y, _ = vmb.vmb_causal_conv_fwd(x, w)
    assert ref.rel(y, ref.conv(d(x), d(w), None)[0]) <= OUT[F32]
    assert vmb.vmb_causal_conv_bwd(x, w, None, dy)["bias"] is None


def test_gradients_against_differences(vmb):
    """Along a random direction, by a central difference of step 2^-7: its truncation is below 2^-14 of the third derivative,
    fp32 outputs off by 2^-21 leave 2^-14 of the sum's size; 2^-9 of the gradient's norm times the direction's covers both."""
    x, w, b, _, dy, _ = make(6, 2, 50, 24, 4, F32)
    got, step = vmb.vmb_causal_conv_bwd(x, w, b, dy), 2.0 ** -7
    for name, i in (("x", 0), ("weight", 1), ("bias", 2)):
        dirs = torch.randn_like((x, w, b)[i])

        def loss(s):
            ins = [x, w, b]
            ins[i] = ins[i] + s * step * dirs
            return (vmb.vmb_causal_conv_fwd(*ins)[0].double() * dy.double()).sum()

        slope = (loss(1) - loss(-1)) / (2 * step)
        want = (got[name].double() * dirs.double()).sum()
        assert abs(float(slope - want)) <= 2.0 ** -9 * float(got[name].norm() * dirs.norm()), name


def test_offsets_beyond_the_tokens_stay_in_range(vmb):
    x, w, b, _, dy, _ = make(7, 1, 20, 16, 4, F32)
    offsets = torch.tensor([0, 8, 90], dtype=torch.int32, device="cuda")
    y, last = vmb.vmb_causal_conv_fwd(x, w, b, offsets=offsets, want_state=True)
    cut = torch.tensor([0, 8, 20], dtype=torch.int32, device="cuda")
    want, wlast = vmb.vmb_causal_conv_fwd(x, w, b, offsets=cut, want_state=True)
    assert torch.equal(y, want) and torch.equal(last, wlast)
    a, c = (vmb.vmb_causal_conv_bwd(x, w, b, dy, offsets=o) for o in (offsets, cut))
    assert all(torch.equal(a[k], c[k]) for k in a)


def test_deterministic(vmb):
    x, w, b, _, dy, _ = make(8, 3, 500, 96, 4, BF16)
    a, c = (vmb.vmb_causal_conv_bwd(x, w, b, dy) for _ in range(2))
    assert all(torch.equal(a[k], c[k]) for k in a)
