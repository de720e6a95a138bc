"""Root-mean-square norm against its definition in 64 bits.

Tolerances: the sum of squares of C terms in fp32, joined over up to 512 threads of 32 values each, is off by less than
2^-24 (32 + 9 + 3) relative, half of that in rstd; with the products 2^-18 covers an element.  bf16 storage adds one rounding of at most 2^-8; e4m3 one of at most 2^-4 of a normal
value, and of 2^-10 below 2^-6 (half its least step)."""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = 2.0 ** -18
CASES = [(5, 96, F32), (1, 1, F32), (7, 192, BF16), (3, 1000, BF16), (2, 4096, F32), (4, 8192, BF16), (2, 8192, F32), (9, 7, BF16), (300, 768, F32),
         (2, 8191, BF16), (33, 385, F32), (130, 33, F32), (1, 1537, BF16), (700, 128, BF16)]


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    return vmb


def make(rows, C, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    return r(rows, C).to(dtype), 1 + 0.3 * r(C), (3 * r(rows, C)).to(dtype), r(rows, C).to(dtype), r(rows, C).to(dtype)


def norm(s, w, eps=1e-6):
    return s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps) * (1.0 if w is None else w)


@pytest.mark.parametrize("rows,C,dtype", CASES)
@pytest.mark.parametrize("residual,weight", [(True, True), (False, True), (True, False)])
def test_forward_and_gradients(vmb, rows, C, dtype, residual, weight):
    x, w, res, dy, dsum = make(rows, C, dtype)
    res, w = res if residual else None, w if weight else None
    y, total, scale, rstd = vmb.vmb_rms_norm_fwd(x, w, res, want_stats=True)
    assert scale is None
    s = x if res is None else total
    if residual:
        assert torch.equal(total, x + res)
    yr = norm(s.double(), w if w is None else w.double())
    assert ((y.double() - yr).abs() <= (TOL + ref.HALF[dtype]) * yr.abs()).all()
    got = vmb.vmb_rms_norm_bwd(s, w, rstd, dy, dsum=dsum if residual else None)
    want = ref.gradients(lambda s, w: (norm(s, w), s), (s, w), (dy, dsum if residual else None))
    # dx = rstd (dn - n mean(dn n)), dn = w dy: the second term is no longer than the first (n is of length sqrt(C) at most, so it is
    # dn's part along n, times at most 1), and what is left of the two can be far smaller than either (C = 1: dn eps rstd^2).  Each
    # is off by 2^-18 of its own length; only the rounding to the storage type goes by the difference.
    terms = float((rstd.double().unsqueeze(1) * dy.double() * (1.0 if w is None else w.double())).norm())
    off = float((got["x"].double().cpu() - want[0]).norm())
    assert off <= 2.0 ** -17 * terms + (2.0 ** -18 + ref.HALF[dtype]) * float(want[0].norm())
    # (sums over up to 700 rows of random sign: a condition of 2^5 at most)
    assert got["weight"] is None if w is None else ref.rel(got["weight"], want[1]) <= 2.0 ** -13


@pytest.mark.parametrize("rows,C,dtype", CASES)
def test_eight_bits(vmb, rows, C, dtype):
    x, w, res, _, _ = make(rows, C, dtype, 2)
    x[0] = 0
    res[0] = 0
    y, total, scale, rstd = vmb.vmb_rms_norm_fwd(x, w, res, bits8=True)
    assert y.dtype == torch.float8_e4m3fn and rstd is None and torch.equal(total, x + res)
    yr = norm(total.double(), w.double())
    want = (yr.abs().amax(1) / 448).clamp(min=2.0 ** -100)
    assert ((scale.double() - want).abs() <= TOL * want).all()
    v = yr / scale.double().unsqueeze(1)
    assert ((y.double() - v).abs() <= (2.0 ** -4 + TOL) * v.abs() + 2.0 ** -10).all()
    assert not y[0].double().any()


def test_unaligned_and_batched(vmb):
    x, w, res, dy, _ = make(9, 64, BF16, 3)
    off = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731 (2 or 4 bytes past 16)
    a, b = vmb.vmb_rms_norm_fwd(x, w, res, want_stats=True), vmb.vmb_rms_norm_fwd(off(x), off(w), off(res), want_stats=True)
    yr = norm(a[1].double(), w.double())
    for t in (a, b):
        assert ((t[0].double() - yr).abs() <= (TOL + 2.0 ** -8) * yr.abs()).all()
    assert torch.equal(a[1], b[1])
    c = vmb.vmb_rms_norm_fwd(x.view(3, 3, 64), w, res.view(3, 3, 64), want_stats=True)
    assert torch.equal(c[0].view(9, 64), a[0]) and torch.equal(c[3].view(9), a[3])
    g, h = (vmb.vmb_rms_norm_bwd(f(a[1]), f(w), a[3], f(dy)) for f in (lambda t: t, off))
    assert ref.rel(h["x"], g["x"]) <= 2.0 ** -8 and ref.rel(h["weight"], g["weight"]) <= 2.0 ** -13


def test_a_row_of_what_is_not_finite_stays_alone(vmb):
    x, w, _, _, _ = make(6, 200, F32, 4)
    x[1, 3], x[4, 7] = float("inf"), float("nan")
    y, _, _, _ = vmb.vmb_rms_norm_fwd(x, w)
    y8, _, scale, _ = vmb.vmb_rms_norm_fwd(x, w, bits8=True)
    for r in (0, 2, 3, 5):
        yr = norm(x[r].double(), w.double())
        assert ((y[r].double() - yr).abs() <= TOL * yr.abs()).all()
        assert (y8[r].double() * scale[r].double() - yr).abs().max() <= (2.0 ** -4 + TOL) * yr.abs().max()
    assert y[4].isnan().all()


def test_gradients_against_differences(vmb):
    """Central difference of step 2^-7 along a direction: truncation and fp32 outputs each below 2^-11 here."""
    x, w, _, dy, _ = make(20, 96, F32, 5)
    _, _, _, rstd = vmb.vmb_rms_norm_fwd(x, w, want_stats=True)
    got, step = vmb.vmb_rms_norm_bwd(x, w, rstd, dy), 2.0 ** -7
    for i, name in enumerate(("x", "weight")):
        way = torch.randn_like((x, w)[i])

        def loss(s):
            t = [x, w]
            t[i] = t[i] + s * step * way
            return (vmb.vmb_rms_norm_fwd(*t)[0].double() * dy.double()).sum()

        slope, want = (loss(1) - loss(-1)) / (2 * step), (got[name].double() * way.double()).sum()
        assert abs(float(slope - want)) <= 2.0 ** -9 * float(got[name].norm() * way.norm()), name
