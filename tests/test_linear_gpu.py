"""The matrix product of a projection against its definition in 64 bits.

Tolerances: products of bf16 or e4m3 values are exact in fp32; a sum of K of them in fp32, in any order, is off by at most K 2^-24
of the sum of magnitudes (the tensor cores may drop bits below 2^-23 of the largest term of a step instead of rounding, the same order).  With terms of
random sign the magnitudes exceed the sums by sqrt(K) in the norm: K^1.5 2^-24 bounds it, K <= 512 here or 1100 (K^1.5 2^-24 = 2^-9); what is
measured lies far below.  The output is rounded once, at most 2^-8."""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def tol(K):
    return 2.0 ** -8 + (K ** 1.5 + 64) * 2.0 ** -24


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    return vmb


def rand(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, device="cuda", generator=g)


def eight(t):
    scale = t.abs().amax(1) / 448
    return (t / scale.unsqueeze(1)).to(E4M3), scale


def product(x, w, bias, act, residual, xs=None, ws=None):
    x, w = x.double(), w.double()
    if xs is not None:
        x, w = x * xs.double().unsqueeze(1), w * ws.double().unsqueeze(1)
    z = x @ w.t()
    if bias is not None:
        z = z + bias.double()
    y = ref.activation(z, act)
    return (y if residual is None else y + residual.double()), z


# many tiles for each SM, with ragged edges
LARGE = [(2500, 200, 2600), (4096, 64, 2056), (1025, 1032, 5000), (3000, 2048, 2304)]
SIZES = [(1, 64, 64), (1, 200, 104), (2, 512, 8), (3, 72, 136), (7, 256, 300), (8, 128, 77), (16, 512, 256), (17, 96, 129), (32, 264, 200), (33, 64, 64),
         (64, 512, 256), (100, 136, 333), (128, 128, 256), (129, 192, 257), (200, 1024, 520), (256, 64, 512), (300, 320, 264), (513, 80, 1000), (1, 1, 1),
         (5, 3, 7), (70, 33, 50), (128, 1100, 40), (1000, 16, 24), (2, 0, 5)]


def close(y, want, K):
    """By the norm, and no element beyond what the sums' terms allow it (outputs are of order one)."""
    assert ref.rel(y, want) <= tol(K)
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + K * 2.0 ** -20 + 2.0 ** -16).all()


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("act,bias,residual", [("none", False, False), ("silu", True, True), ("gelu", True, False), ("none", True, True)])
def test_bf16(vmb, M, K, N, act, bias, residual):
    r = rand(M * 7 + K + N)
    x, w = r(M, K).to(BF16), (r(N, K) / max(K, 1) ** 0.5).to(BF16)
    b, res = r(N) if bias else None, r(M, N).to(BF16) if residual else None
    y, pre = vmb.vmb_linear_fwd(x, w, b, act=act, residual=res, want_pre=True)
    want, z = product(x, w, b, act, res)
    close(y, want, K)
    close(pre, z, K)
    assert torch.equal(vmb.vmb_linear_fwd(x, w, b, act=act, residual=res)[0], y)


@pytest.mark.parametrize("M,K,N", LARGE)
def test_many_tiles(vmb, M, K, N):
    r = rand(M + K + N)
    x, w, b, res, dy = r(M, K).to(BF16), (r(N, K) / K ** 0.5).to(BF16), r(N), r(M, N).to(BF16), r(M, N).to(BF16)
    y, pre = vmb.vmb_linear_fwd(x, w, b, act="gelu", residual=res, want_pre=True)
    want, z = product(x, w, b, "gelu", res)
    close(y, want, K)
    close(pre, z, K)
    (x8, xs), (w8, ws) = eight(r(M, K // 16 * 16)), eight(r(N, K // 16 * 16) / K ** 0.5)
    close(vmb.vmb_linear_fwd(x8, w8, b, act="silu", x_scale=xs, weight_scale=ws)[0], product(x8, w8, b, "silu", None, xs, ws)[0], K)
    if N % 8 == 0:
        d = vmb.vmb_linear_bwd(x, w, dy, want_bias=True)
        assert ref.rel(d["x"], dy.double() @ w.double()) <= tol(N) and ref.rel(d["weight"], dy.double().t() @ x.double()) <= tol(M)
        # a mistake in one tile: no element is off by more than its rounding and a sum's 2^-20 of its terms (dx: N terms of 1 / sqrt(K); dweight: M of one)
        dx, dw = dy.double() @ w.double(), dy.double().t() @ x.double()
        assert ((d["x"].double() - dx).abs() <= 2.0 ** -8 * dx.abs() + N * 2.0 ** -20).all()
        assert ((d["weight"].double() - dw).abs() <= 2.0 ** -8 * dw.abs() + M * 2.0 ** -20).all()
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK


@pytest.mark.parametrize("M,K,N", [s for s in SIZES if s[1]])
@pytest.mark.parametrize("act,bias,residual", [("none", False, False), ("gelu", True, True)])
def test_eight_bits(vmb, M, K, N, act, bias, residual):
    r = rand(M * 5 + K + N)
    (x, xs), (w, ws) = eight(r(M, K)), eight(r(N, K) / K ** 0.5)
    b, res = r(N) if bias else None, r(M, N).to(BF16) if residual else None
    y, _ = vmb.vmb_linear_fwd(x, w, b, act=act, residual=res, x_scale=xs, weight_scale=ws)
    close(y, product(x, w, b, act, res, xs, ws)[0], K)


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_gradients(vmb, M, K, N, act):
    r = rand(M * 3 + K + N)
    x, w, dy = r(M, K).to(BF16), (r(N, K) / max(K, 1) ** 0.5).to(BF16), r(M, N).to(BF16)
    pre = r(M, N).to(BF16) if act != "none" else None
    got = vmb.vmb_linear_bwd(x, w, dy, pre, act=act, want_bias=True)
    dz = dy.double()
    if pre is not None:
        p = pre.double().requires_grad_()
        dz, = torch.autograd.grad(ref.activation(p, act), p, dz)
    # dZ is rounded before the products (2^-8), their sums once more
    more = 0.0 if pre is None else 2.0 ** -8
    assert ref.rel(got["x"], dz @ w.double()) <= tol(N) + more
    assert ref.rel(got["weight"], dz.t() @ x.double()) <= tol(M) + more
    assert ref.rel(got["bias"], dz.sum(0)) <= 2.0 ** -14
    only = vmb.vmb_linear_bwd(x, w, dy, pre, act=act, want_x=False)
    assert only["x"] is None and only["bias"] is None and torch.equal(only["weight"], got["weight"])


@pytest.mark.parametrize("M,K,N,ld", [(40, 64, 72, 160), (200, 256, 128, 264), (9, 40, 33, 43), (3, 512, 64, 1024)])
def test_strided_rows_of_x(vmb, M, K, N, ld):
    r = rand(5)
    wide, w, dy = r(M, ld).to(BF16), (r(N, K) / K ** 0.5).to(BF16), r(M, N).to(BF16)
    x = wide[:, ld - K:]
    assert torch.equal(vmb.vmb_linear_fwd(x, w)[0], vmb.vmb_linear_fwd(x, w)[0])
    close(vmb.vmb_linear_fwd(x, w)[0], product(x, w, None, "none", None)[0], K)
    assert ref.rel(vmb.vmb_linear_bwd(x, w, dy)["weight"], dy.double().t() @ x.double()) <= tol(M)


def test_unaligned_operands(vmb):
    r = rand(6)
    off = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    for M in (2, 20, 150):
        x, w, res = off(r(M, 64).to(BF16)), off((r(96, 64) / 8).to(BF16)), off(r(M, 96).to(BF16))
        close(vmb.vmb_linear_fwd(x, w, residual=res)[0], product(x, w, None, "none", res)[0], 64)
        close(vmb.vmb_linear_fwd(x.clone(), w.clone(), residual=res)[0], product(x, w, None, "none", res)[0], 64)


def test_batch_dimensions(vmb):
    r = rand(7)
    x, w = r(3, 5, 64).to(BF16), r(40, 64).to(BF16)
    y, pre = vmb.vmb_linear_fwd(x, w, act="silu", want_pre=True)
    flat, _ = vmb.vmb_linear_fwd(x.view(15, 64), w, act="silu")
    assert y.shape == (3, 5, 40) and torch.equal(y.view(15, 40), flat)
    d = vmb.vmb_linear_bwd(x, w, y, pre, act="silu", want_bias=True)
    assert d["x"].shape == x.shape and d["weight"].shape == w.shape and d["bias"].shape == (40,)


def test_activation_far_out(vmb):
    """GELU and SiLU keep their digits where they are small: rounded once from the definition (2^-8) and 2^-12 for the function."""
    z = torch.linspace(-12, 12, 4096, device="cuda")
    x, w = torch.ones(1, 8, device="cuda", dtype=BF16), torch.zeros(4096, 8, device="cuda", dtype=BF16)
    for M in (1, 40, 200):
        for act in ("silu", "gelu"):
            y = vmb.vmb_linear_fwd(x.expand(M, 8).contiguous(), w, z, act=act)[0]
            want = ref.activation(z.double(), act).expand(M, -1)
            assert ((y.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -12) * want.abs() + 1e-37).all(), act


def test_what_is_not_finite_stays_in_its_row(vmb):
    r = rand(8)
    for M in (4, 40, 200):
        x, w = r(M, 128).to(BF16), r(72, 128).to(BF16)
        x[1, 5] = float("nan")
        y = vmb.vmb_linear_fwd(x, w)[0]
        rest = [i for i in range(M) if i != 1]
        assert y[1].isnan().all()
        close(y[rest], product(x[rest], w, None, "none", None)[0], 128 * 16)  # (weights of order one: sums of order 2^3.5)


def test_activations_of_what_is_not_finite(vmb):
    bias = torch.tensor([float("inf"), float("-inf"), float("nan"), 0.0, -300.0, 300.0, -0.0, 3.0], device="cuda")
    for M in (1, 40, 200):
        x, w = torch.zeros(M, 8, device="cuda", dtype=BF16), torch.zeros(8, 8, device="cuda", dtype=BF16)
        for act in ("silu", "gelu"):
            y = vmb.vmb_linear_fwd(x, w, bias, act=act)[0].float()
            assert (y[:, 0] == float("inf")).all() and y[:, 2].isnan().all() and not y[:, [3, 4, 6]].any() and (y[:, 5] == 300).all(), act


def test_rows_that_tensor_copies_refuse(vmb, force_plan):
    """The kernel of any strides at sizes that the others take."""
    r = rand(10)
    x, w, b, res, dy = r(300, 264).to(BF16), (r(520, 264) / 16).to(BF16), r(520), r(300, 520).to(BF16), r(300, 520).to(BF16)
    force_plan.refuse_tensor_maps()
    close(vmb.vmb_linear_fwd(x, w, b, act="silu", residual=res)[0], product(x, w, b, "silu", res)[0], 264)
    d = vmb.vmb_linear_bwd(x, w, dy)
    assert ref.rel(d["x"], dy.double() @ w.double()) <= tol(520) and ref.rel(d["weight"], dy.double().t() @ x.double()) <= tol(300)


def test_rows_of_x_all_the_same(vmb):
    """x expanded from one row: a stride of zero between its rows."""
    r = rand(11)
    x, w = r(1, 64).to(BF16), (r(72, 64) / 8).to(BF16)
    for M in (5, 50, 200):
        y = vmb.vmb_linear_fwd(x.expand(M, 64), w)[0]
        close(y, product(x.expand(M, 64), w, None, "none", None)[0], 64)


def test_empty(vmb):
    r = rand(9)
    assert vmb.vmb_linear_fwd(r(0, 8).to(BF16), r(4, 8).to(BF16))[0].shape == (0, 4)
    d = vmb.vmb_linear_bwd(r(0, 8).to(BF16), r(4, 8).to(BF16), r(0, 4).to(BF16), want_bias=True)
    assert not d["weight"].any() and not d["bias"].any()
