"""The selective scan over tokens against its definition in 64 bits: dense and packed sequences, states, gate, gradients,
steps.

Tolerances: a token's decay is off by about 2^-22 (the exponential) plus 2^-23 |dt A| (its argument), its input by 2^-21
(the softplus); over T tokens that adds up to 4 (T + 8) 2^-24 relative to the sum of the terms' magnitudes, which exceeds the sums by
less than the 4 in the norm of a whole tensor: 2^-22 (T + 8) 4 is the tolerance.  bf16 storage adds one rounding, 2^-8."""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def tol(T, dtype=F32):
    return 2.0 ** -20 * (T + 8) + (2.0 ** -8 if dtype == BF16 else 0.0)


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    return vmb


def make(seed, B, T, D, N, dtype, gate=True, half=False, n=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    n = B if n is None else n
    if half:
        x, z = r(B, T, 2 * D).to(dtype).split(D, -1)
        _, Bm, Cm = r(B, T, 5 + 2 * N).to(dtype).split([5, N, N], -1)
    else:
        x, z, Bm, Cm = r(B, T, D).to(dtype), r(B, T, D).to(dtype), r(B, T, N).to(dtype), r(B, T, N).to(dtype)
    ins = [x, r(B, T, D).to(dtype), -torch.arange(1, N + 1, device="cuda") * torch.rand(D, N, device="cuda", generator=g), Bm, Cm, r(D),
           r(D) - 2, z if gate else None]
    return ins, r(n, D, N), r(B, T, D).to(dtype), r(n, D, N)


def d(ts):
    return [None if t is None else t.double().cpu() for t in ts]


NAMES = ("x", "delta", "A", "B", "C", "Dskip", "delta_bias", "z")
CASES = [(2, 37, 24, 16, F32, True, False), (1, 1, 8, 16, BF16, True, False), (3, 5, 7, 3, F32, False, True), (2, 130, 96, 16, BF16, True, True),
         (1, 300, 72, 8, F32, True, False), (2, 64, 64, 4, BF16, False, False), (1, 200, 130, 16, F32, False, False), (2, 0, 16, 16, F32, True, False),
         (1, 129, 65, 13, BF16, True, True), (1, 450, 40, 16, BF16, True, False), (1, 63, 33, 1, F32, True, False), (2, 65, 64, 6, F32, True, True)]


@pytest.mark.parametrize("B,T,D,N,dtype,gate,half", CASES)
@pytest.mark.parametrize("state", [False, True])
def test_forward_and_gradients(vmb, B, T, D, N, dtype, gate, half, state):
    ins, init, dy, dlast = make(1, B, T, D, N, dtype, gate, half)
    init, dlast = (init, dlast) if state else (None, None)
    y, last, saved = vmb.vmb_token_scan_fwd(*ins, initial_state=init, want_state=state, want_saved=True)
    yr, lr = ref.scan(*d(ins), *d([init]))
    assert ref.rel(y, yr) <= tol(T, dtype)
    if state:
        assert ref.rel(last, lr) <= tol(T)
    got = vmb.vmb_token_scan_bwd(*ins, dy, saved, dfinal_state=dlast, want_initial=state)
    want = ref.gradients(lambda *t: ref.scan(*t), (*ins, init), (dy, dlast))
    for name, w in zip((*NAMES, "initial_state"), want):
        if w is None:
            assert name == "z" and got[name] is None or not state
        elif not T and name != "initial_state":
            assert not got[name].any()
        else:
            assert ref.rel(got[name], w) <= tol(T, got[name].dtype), name
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK


PACKED = [(3, [0, 1, 2, 3, 150, 0, 17, 64], 5), (0, [1], 0), (0, [70, 0, 0, 133], 0), (7, [0, 0], 9), (0, [64, 128, 63, 65], 16)]


@pytest.mark.parametrize("lead,lens,tail", PACKED)
@pytest.mark.parametrize("D,N,dtype", [(24, 16, F32), (40, 16, BF16), (5, 3, BF16), (72, 8, F32)])
def test_packed(vmb, lead, lens, tail, D, N, dtype):
    at = [lead]
    for n in lens:
        at.append(at[-1] + n)
    T, most = at[-1] + tail, max(lens)
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    ins, init, dy, dlast = make(2, 1, T, D, N, dtype, n=len(lens))
    y, last, saved = vmb.vmb_token_scan_fwd(*ins, initial_state=init, offsets=offsets, want_state=True, want_saved=True,
                                            y=torch.full((1, T, D), 7.0, device="cuda").to(dtype))
    yr, lr = ref.scan(*d(ins), init.double().cpu(), offsets)
    assert ref.rel(y, yr) <= tol(most, dtype) and ref.rel(last, lr) <= tol(most)
    assert not y[:, :lead].any() and not y[:, at[-1]:].any()
    got = vmb.vmb_token_scan_bwd(*ins, dy, saved, dfinal_state=dlast, offsets=offsets, want_initial=True)
    want = ref.gradients(lambda *t: ref.scan(*t, offsets), (*ins, init), (dy, dlast))
    for name, w in zip((*NAMES, "initial_state"), want):
        assert ref.rel(got[name], w) <= tol(most, got[name].dtype), name
    for name in ("x", "delta", "B", "C", "z"):
        assert not got[name][:, :lead].any() and not got[name][:, at[-1]:].any(), name
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK


def test_long_chain_in_segments(vmb):
    """One sequence over few channels is cut into segments; the reference is the same call on its parts, one after the other."""
    ins, init, _, _ = make(3, 1, 3000, 48, 16, F32)
    y, last, _ = vmb.vmb_token_scan_fwd(*ins, initial_state=init, want_state=True)
    parts, h = [], init
    for t0 in range(0, 3000, 100):  # (100 tokens are never cut)
        part = [t if t is None or t.dim() < 3 else t[:, t0:t0 + 100] for t in ins]
        o, h, _ = vmb.vmb_token_scan_fwd(*part, initial_state=h, want_state=True)
        parts.append(o)
    # both are within 4 (T + 8) 2^-22 of the truth over the memory of the slowest state, about 1 / (dt |A|) < 2^10 tokens
    assert ref.rel(y, torch.cat(parts, 1)) <= 2 * tol(1024) and ref.rel(last, h) <= 2 * tol(1024)


@pytest.mark.parametrize("B,T,D,N,dtype,gate,slots", [(5, 1, 40, 16, BF16, True, True), (3, 3, 7, 3, F32, False, True), (4, 2, 264, 8, F32, True, False),
                                                      (1, 6, 100, 16, BF16, True, True), (2, 1, 33, 5, F32, True, False), (3, 1, 8, 4, BF16, False, True)])
def test_steps(vmb, B, T, D, N, dtype, gate, slots):
    ins, _, _, _ = make(4, B, T, D, N, dtype, gate)
    pool = torch.randn(B + 4, D, N, device="cuda")
    old, at = pool.clone(), torch.arange(B, dtype=torch.int32)
    if slots:
        at = torch.randperm(B + 4, generator=torch.Generator().manual_seed(1))[:B].to(torch.int32)
        if B > 1:
            at[1] = -1
    y = vmb.vmb_token_scan_step(*ins, pool, slots=at.cuda() if slots else None)
    used = [i for i in range(B) if at[i] >= 0]
    yr, lr = ref.scan(*[t if t is None or t.dim() < 3 else t[used] for t in d(ins)], old[at[used].long()].double().cpu())
    assert ref.rel(y[used], yr) <= tol(T, dtype)
    assert ref.rel(pool[at[used].long()], lr) <= tol(T)
    rest = [i for i in range(B + 4) if i not in at[used].tolist()]
    assert torch.equal(pool[rest], old[rest])
    assert not y[[i for i in range(B) if at[i] < 0]].any()


@pytest.mark.parametrize("B,T,D,N,dtype", [(3, 2, 40, 16, BF16), (2, 1, 24, 8, F32), (5, 1, 33, 16, F32)])
def test_steps_of_strided_rows(vmb, B, T, D, N, dtype):
    """Parts of wider rows, B and C from an odd place in theirs."""
    ins, init, _, _ = make(10, B, T, D, N, dtype, half=True)
    state = init.clone()
    y = vmb.vmb_token_scan_step(*ins, state)
    yr, lr = ref.scan(*d(ins), *d([init]))
    assert ref.rel(y, yr) <= tol(T, dtype) and ref.rel(state, lr) <= tol(T)
    dense = [t if t is None or t.dim() < 3 else t.contiguous() for t in ins]
    again = init.clone()
    assert torch.equal(vmb.vmb_token_scan_step(*dense, again), y) and torch.equal(again, state)


def test_no_softplus_no_skip_no_bias(vmb):
    ins, init, dy, _ = make(5, 2, 50, 24, 16, F32)
    ins[1], ins[5], ins[6] = ins[1].abs() * 0.1, None, None
    y, _, saved = vmb.vmb_token_scan_fwd(*ins, softplus=False, want_saved=True)
    yr, _ = ref.scan(*d(ins), softplus=False)
    assert ref.rel(y, yr) <= tol(50)
    got = vmb.vmb_token_scan_bwd(*ins, dy, saved, softplus=False)
    want = ref.gradients(lambda *t: ref.scan(*t, softplus=False), ins, (dy,))
    for name, w in zip(NAMES, want):
        assert got[name] is None if w is None else ref.rel(got[name], w) <= tol(50), name


def test_gradients_against_differences(vmb):
    """Along a random direction, by a central difference of step 2^-8: truncation below 2^-13 here, outputs off by 2^-20 leave
    2^-12 of the sum's size; 2^-8 of the gradient's norm times the direction's covers both."""
    ins, _, dy, _ = make(6, 2, 60, 24, 16, F32)
    _, _, saved = vmb.vmb_token_scan_fwd(*ins, want_saved=True)
    got, step = vmb.vmb_token_scan_bwd(*ins, dy, saved), 2.0 ** -8
    for i, name in enumerate(NAMES):
        way = torch.randn_like(ins[i])

        def loss(s):
            t = list(ins)
            t[i] = t[i] + s * step * way
            return (vmb.vmb_token_scan_fwd(*t)[0].double() * dy.double()).sum()

        slope, want = (loss(1) - loss(-1)) / (2 * step), (got[name].double() * way.double()).sum()
        assert abs(float(slope - want)) <= 2.0 ** -8 * float(got[name].norm() * way.norm()), name


def test_bad_offsets_are_cut_and_reported(vmb):
    ins, _, dy, _ = make(7, 1, 100, 24, 16, F32)
    offsets = torch.tensor([0, 40, 900], dtype=torch.int32, device="cuda")
    y, last, saved = vmb.vmb_token_scan_fwd(*ins, offsets=offsets, want_state=True, want_saved=True)
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_ERR_BOUNDS
    cut = torch.tensor([0, 40, 100], dtype=torch.int32, device="cuda")
    want, wlast, wsaved = vmb.vmb_token_scan_fwd(*ins, offsets=cut, want_state=True, want_saved=True)
    assert torch.equal(y, want) and torch.equal(last, wlast) and vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK
    a, b = vmb.vmb_token_scan_bwd(*ins, dy, saved, offsets=offsets), vmb.vmb_token_scan_bwd(*ins, dy, wsaved, offsets=cut)
    assert all(torch.equal(a[k], b[k]) for k in NAMES)
    vmb.vmb_read_status(vmb.layer_workspace())


def test_large_steps_forget_and_nan_stays_in_its_sequence(vmb):
    ins, _, _, _ = make(8, 3, 70, 24, 16, F32)
    ins[1][0, 20] = 1e4  # exp(dt A) is 0: what was before is gone
    ins[0][1, 10] = float("nan")
    y, last, _ = vmb.vmb_token_scan_fwd(*ins, want_state=True)
    yr, lr = ref.scan(*d(ins))
    for b in (0, 2):
        assert ref.rel(y[b], yr[b]) <= tol(70) and ref.rel(last[b], lr[b]) <= tol(70)
    assert ref.rel(y[1, :10], yr[1, :10]) <= tol(70) and y[1, 10:].isnan().all()


def test_deterministic(vmb):
    ins, _, dy, _ = make(9, 2, 500, 96, 16, BF16)
    _, _, saved = vmb.vmb_token_scan_fwd(*ins, want_saved=True)
    a, b = (vmb.vmb_token_scan_bwd(*ins, dy, saved) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in NAMES)
