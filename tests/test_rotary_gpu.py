"""Rotary positions with several axes against the turn in 64 bits.  fp32: an angle's sine is off by at most about
2^-22, a turned value by three roundings more: 1e-6 of the vector's length allowed.  bf16: one rounding, 2^-9 at most."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def reference(x, freq, at, sections, interleaved, inverse):
    """at [axes, B, T]"""
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    a = (at.double()[axis].permute(1, 2, 0) * freq.double()).unsqueeze(2)
    cos, sin = torch.cos(a), torch.sin(a) * (-1 if inverse else 1)
    x, y, P = x.double(), x.double().clone(), sum(sections)
    one, two = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    y[..., one] = x[..., one] * cos - x[..., two] * sin
    y[..., two] = x[..., two] * cos + x[..., one] * sin
    return y


def grid_places(grid, B):
    at = torch.cartesian_prod(*[torch.arange(n) for n in grid]).view(-1, len(grid)).t()
    return at.unsqueeze(1).expand(len(grid), B, at.shape[1])


def check(got, want, dtype):
    got = got.double().cpu()
    limit = 1e-6 if dtype == torch.float32 else 2 ** -8
    assert ((got - want).abs() <= limit * want.abs() + 1e-6 * want.abs().max() + 1e-30).all()


CASES = [  # B, grid, Hq, Hk, D, sections
    (1, (1,), 1, 1, 2, (1,)), (2, (7, 5), 3, 1, 64, (16, 16)), (1, (3, 4, 5), 2, 2, 96, (8, 14, 14)), (2, (33,), 1, 1, 13, (5,)),
    (1, (2, 3, 2, 3), 2, 1, 40, (4, 0, 8, 8)), (3, (9, 11), 4, 2, 128, (32, 32)), (1, (6, 6), 2, 2, 72, (12, 24)),
    (2, (5, 3), 1, 2, 36, (3, 6)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_grid_and_positions(case, interleaved, inverse, dtype):
    import paper_2412_16602_gb300 as vmb
    B, grid, Hq, Hk, D, sections = case
    T, dt = math.prod(grid), TYPES[dtype]
    gen = torch.Generator().manual_seed(D)
    q, k = torch.randn(B, T, Hq, D, generator=gen).to(dt), torch.randn(B, T, Hk, D, generator=gen).to(dt)
    freq = torch.rand(sum(sections), generator=gen)
    kw = dict(sections=sections, interleaved=interleaved, inverse=inverse)
    at = grid_places(grid, B)
    a, b = vmb.vmb_rotary_fwd(q.cuda(), k.cuda(), freq.cuda(), grid=grid, **kw)
    check(a, reference(q, freq, at, sections, interleaved, inverse), dt)
    check(b, reference(k, freq, at, sections, interleaved, inverse), dt)
    c, d = vmb.vmb_rotary_fwd(q.cuda(), k.cuda(), freq.cuda(), at.to(torch.int32).contiguous().cuda(), **kw)
    assert torch.equal(a, c) and torch.equal(b, d)
    alone, none = vmb.vmb_rotary_fwd(q.cuda(), None, freq.cuda(), grid=grid, **kw)
    assert none is None and torch.equal(alone, a)


def test_far_and_negative_positions():
    """The angle's rounding does not grow with the position."""
    import paper_2412_16602_gb300 as vmb
    places = [0, -1, 4096, -70001, 1 << 20, (1 << 24) + 1, 2147483647, -2147483648]
    at = torch.tensor(places, dtype=torch.int32).view(1, 1, -1)
    gen = torch.Generator().manual_seed(1)
    q = torch.randn(1, len(places), 2, 16, generator=gen)
    freq = torch.tensor([1.0, 0.7310585786300049, 0.1, 0.01, 1e-3, 1e-4, 3.0, 1e-8])
    got, _ = vmb.vmb_rotary_fwd(q.cuda(), None, freq.cuda(), at.cuda(), sections=(8,))
    want = reference(q, freq, at, (8,), False, False)
    # hi + lo carries 48 bits of the angle: 2^31 * 2^-48 at the farthest
    assert ((got.double().cpu() - want).abs().amax((0, 2, 3)) <= 1e-5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_odd_and_in_place(dtype):
    import paper_2412_16602_gb300 as vmb
    dt = TYPES[dtype]
    torch.manual_seed(8)
    row = torch.randn(2, 12, 3 * 64 + 64 + 1, device="cuda").to(dt)
    q, k = row[..., :192].view(2, 12, 3, 64), row[..., 192:256].view(2, 12, 1, 64)
    freq = torch.rand(32, device="cuda")
    kw = dict(sections=(16, 16), grid=(3, 4))
    a, b = vmb.vmb_rotary_fwd(q, k, freq, **kw)
    qd, kd = q.contiguous(), k.contiguous()
    c, d = vmb.vmb_rotary_fwd(qd, kd, freq, **kw)
    assert torch.equal(a, c) and torch.equal(b, d)
    vmb.vmb_rotary_fwd(qd, kd, freq, q_out=qd, k_out=kd, **kw)
    assert torch.equal(qd, a) and torch.equal(kd, b)
    back, _ = vmb.vmb_rotary_fwd(a, None, freq, inverse=True, **kw)
    assert (back.float() - q.float()).abs().max().item() <= (1e-5 if dtype == "f32" else 0.06)
    with pytest.raises(vmb.VmbError):
        vmb.vmb_rotary_fwd(torch.as_strided(row, (2, 12, 1, 64), (12 * 257, 257, 64, 1)), None, freq,
                           q_out=torch.as_strided(row, (2, 12, 1, 64), (768, 64, 64, 1)), **kw)


def test_refusals_and_empty():
    import paper_2412_16602_gb300 as vmb
    q, freq = torch.zeros(1, 6, 1, 16, device="cuda"), torch.ones(4, device="cuda")
    for kw in (dict(sections=(4,)), dict(sections=(5,), grid=(6,)), dict(sections=(2, 2), grid=(6,)), dict(sections=()),
               dict(sections=(1, 1, 1, 1, 0), grid=(6, 1, 1, 1, 1))):
        with pytest.raises(ValueError):
            vmb.vmb_rotary_fwd(q, None, freq, **kw)
    for kw in (dict(sections=(4,), grid=(5,)), dict(sections=(2, 2), grid=(2, 2))):
        with pytest.raises(vmb.VmbError):
            vmb.vmb_rotary_fwd(q, None, freq, **kw)
    with pytest.raises(vmb.VmbError):
        vmb.vmb_rotary_fwd(q, None, torch.ones(9, device="cuda"), sections=(9,), grid=(6,))
    with pytest.raises(ValueError):
        vmb.vmb_rotary_fwd(q, q[:, :3], freq, sections=(4,), grid=(6,))
    with pytest.raises(TypeError):
        vmb.vmb_rotary_fwd(q.half(), None, freq, sections=(4,), grid=(6,))
    out, _ = vmb.vmb_rotary_fwd(q[:, :0], None, freq, sections=(4,), grid=(0,))
    assert out.shape == (1, 0, 1, 16)
