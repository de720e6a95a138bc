"""The scan over tokens and its gradients over thousands of tokens, cut into dozens of segments, against the definition in 64 bits.

Tolerances: A is at most -1/2 and the mean step size above 0.2, so that a state remembers some 1 / (0.2 / 2) = 10 tokens.  A token's decay is off by 2^-22 (the
exponential) and 2^-23 |dt A| (its argument), so over its memory a state by 2^4 2^-22 at most, 2^-18; the input, the gate and the sums over the states add
2^-20 each, and the sums' terms, of random sign, exceed them by less than 4 in the norm: 2^-16 for outputs and states.  A gradient goes through the adjoint,
of the same memory, and the states: twice as much; sums over tokens (A, D, bias) have terms that are each off by that much, of random sign: 2^-14 for
gradients.  bf16 storage adds one rounding, 2^-8."""
import pytest
import torch

from tests import layer_reference as ref
from tests.test_token_scan_gpu import BF16, F32, NAMES, d

pytestmark = pytest.mark.gpu


def make(B, T, D, N, dtype, gate, n):
    g = torch.Generator(device="cuda").manual_seed(T + D)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    A = -torch.arange(1, N + 1, device="cuda") * (0.5 + 0.5 * torch.rand(D, N, device="cuda", generator=g))
    ins = [r(B, T, D).to(dtype), r(B, T, D).to(dtype), A, r(B, T, N).to(dtype), r(B, T, N).to(dtype), r(D), 0.3 * r(D) - 1.5, r(B, T, D).to(dtype) if gate else None]
    return ins, r(n, D, N), r(B, T, D).to(dtype), r(n, D, N)


@pytest.mark.parametrize("B,T,D,N,dtype,gate,lens", [(1, 3000, 48, 16, F32, True, None), (2, 1500, 65, 8, F32, True, None), (1, 2500, 40, 16, BF16, True, None),
                                                     (1, 4000, 24, 4, F32, False, None), (1, 3100, 64, 16, F32, True, [1300, 0, 1, 900, 899]),
                                                     (1, 2600, 72, 16, BF16, True, [64, 2000, 500]), (1, 2000, 700, 5, F32, True, None)])
def test_long(B, T, D, N, dtype, gate, lens):
    import paper_2412_16602_gb300 as vmb
    offsets = None
    if lens:
        offsets = torch.tensor([0, *torch.tensor(lens).cumsum(0)], dtype=torch.int32, device="cuda")
    ins, init, dy, dlast = make(B, T, D, N, dtype, gate, len(lens) if lens else B)
    y, last, saved = vmb.vmb_token_scan_fwd(*ins, initial_state=init, offsets=offsets, want_state=True, want_saved=True)
    leaves = [None if t is None else t.double().cpu().requires_grad_() for t in (*ins, init)]
    yr, lr = ref.scan(*leaves, None if offsets is None else offsets.cpu())
    half = ref.HALF[dtype] if dtype == BF16 else 0.0
    assert ref.rel(y, yr.detach()) <= 2.0 ** -16 + half and ref.rel(last, lr.detach()) <= 2.0 ** -16
    # segment by segment: no stretch of 64 tokens is off by more than four times the whole's tolerance of the whole's mean size
    at = (y.double().cpu() - yr.detach()).reshape(-1, D)
    mean = float(yr.detach().norm()) / (B * T) ** 0.5
    assert all(float(at[t:t + 64].norm()) <= 4 * (2.0 ** -16 + half) * mean * 8 for t in range(0, B * T, 64))
    live = [t for t in leaves if t is not None]
    grads = iter(torch.autograd.grad((yr * dy.double().cpu()).sum() + (lr * dlast.double().cpu()).sum(), live))
    got = vmb.vmb_token_scan_bwd(*ins, dy, saved, dfinal_state=dlast, offsets=offsets, want_initial=True)
    for name, t in zip((*NAMES, "initial_state"), leaves):
        if t is None:
            assert got[name] is None
        else:
            assert ref.rel(got[name], next(grads)) <= 2.0 ** -14 + (ref.HALF[BF16] if got[name].dtype == BF16 else 0.0), name
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK
