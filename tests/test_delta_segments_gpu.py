"""Chains that are cut into segments (few sequences and heads) against the recurrence in 64 bits: odd numbers of chunks and
segments, keys and values that fill no tile, states on both ends.

Tolerances (2-norm of the difference over that of the reference): those of an uncut chain, since a value passes one more fp32
product per segment (2^-24 of it, at most 40 segments, decaying): fp32 2e-5; bf16 1e-2, fp32 states of bf16 inputs 4e-5."""
import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [  # B, T, Hk, Hv, Dk, Dv
    (1, 256, 1, 1, 64, 64), (1, 513, 1, 2, 100, 130), (1, 600, 1, 1, 40, 33), (2, 900, 1, 2, 9, 5), (1, 1000, 2, 2, 65, 7),
    (1, 385, 1, 1, 128, 264), (1, 2600, 1, 1, 17, 24), (4, 330, 3, 9, 64, 64),
]


def check(got, want, limit, what):
    got = got.double().cpu()
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    assert (got - want).norm().item() <= limit * want.norm().item() + 1e-12, what


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_segments(size, dtype):
    import paper_2412_16602_gb300 as vmb
    dt, (B, T, Hk, Hv, Dk, Dv) = TYPES[dtype], size
    rest, state = (2e-5, 2e-5) if dtype == "f32" else (1e-2, 4e-5)
    x = ref.inputs(*size, seed=sum(size) + 1, dtype=dt)
    gen = torch.Generator().manual_seed(21)
    init, dfinal = torch.randn(B, Hv, Dk, Dv, generator=gen) * 0.3, torch.randn(B, Hv, Dk, Dv, generator=gen)
    do = torch.randn(B, T, Hv, Dv, generator=gen).to(dt)
    o, S, _ = ref.forward(*x, init)
    d = ref.backward(*x, do, init, dfinal)
    c = [t.cuda() for t in x]
    go, gS, saved = vmb.vmb_delta_rule_fwd(*c, initial_state=init.cuda(), want_state=True, want_saved=True)
    gd = vmb.vmb_delta_rule_bwd(*c, do.cuda(), saved, dfinal_state=dfinal.cuda(), want_initial=True)
    check(go, o, rest, "o")
    check(gS, S, state, "final state")
    for n in ("q", "k", "v", "g", "beta"):
        check(gd[n], d[n], rest * (3 if n == "g" else 1), n)  # dg is a difference of such sums
    check(gd["initial_state"], d["initial_state"], state, "initial state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_sequences_of_other_lengths_than_the_longest(dtype):
    import paper_2412_16602_gb300 as vmb
    dt, lens = TYPES[dtype], (700, 0, 64, 321, 1)
    total = sum(lens)
    x = ref.inputs(1, total, 1, 1, 40, 72, 31, dt)
    gen = torch.Generator().manual_seed(22)
    init = torch.randn(len(lens), 1, 40, 72, generator=gen) * 0.3
    at = [sum(lens[:i]) for i in range(len(lens) + 1)]
    go, gS = vmb.vmb_delta_rule_fwd(*[t.cuda() for t in x], initial_state=init.cuda(), want_state=True,
                                    offsets=torch.tensor(at, dtype=torch.int32, device="cuda"), max_len=max(lens))[:2]
    for i, n in enumerate(lens):
        o, S, _ = ref.forward(*[t[:, at[i]:at[i] + n] for t in x], init[i:i + 1])
        check(go[:, at[i]:at[i] + n], o, 2e-5 if dtype == "f32" else 1e-2, f"o {i}")
        check(gS[i:i + 1], S, 2e-5 if dtype == "f32" else 4e-5, f"state {i}")
