"""Products whose contraction is split: the parts' sums are kept in fp32 and a second launch joins them and does what the epilogue does.  Against the
definition in 64 bits, at the tolerances of the product's other tests (K terms of random sign)."""
import ctypes

import pytest
import torch

from tests import layer_reference as ref
from tests.test_linear_gpu import BF16, close, eight, product, rand, tol

pytestmark = pytest.mark.gpu
# rows of whole vectors of eight outputs, and odd ones, which the parts and the join take one by one
SIZES = [(64, 2048, 1003), (64, 2048, 1000), (40, 4096, 512), (100, 4096, 77), (128, 2048, 256), (33, 2560, 8), (200, 4096, 136), (65, 4096, 1)]
EPILOGUES = [("none", False, False, False), ("gelu", True, True, True), ("silu", True, False, True), ("none", True, True, False)]


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    vmb.lib.vmb_testing_linear_plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_void_p]
    return vmb


def parts(vmb, M, K, N, bits8=False):
    out = (ctypes.c_int * 2)()
    assert vmb.lib.vmb_testing_linear_plan(M, N, K, int(bits8), out) == 0
    return out[1]


def off(t):
    """The same values 2 bytes past a multiple of 16."""
    return torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("act,bias,residual,want_pre", EPILOGUES)
def test_bf16(vmb, M, K, N, act, bias, residual, want_pre):
    assert parts(vmb, M, K, N) > 1
    r = rand(M + 3 * K + N)
    x, w = r(M, K).to(BF16), (r(N, K) / K ** 0.5).to(BF16)
    b, res = r(N) if bias else None, r(M, N).to(BF16) if residual else None
    want, z = product(x, w, b, act, res)
    y, pre = vmb.vmb_linear_fwd(x, w, b, act=act, residual=res, want_pre=want_pre)
    close(y, want, K)
    if want_pre:
        close(pre, z, K)
    # outputs and residual that do not start on 16 bytes
    out = off(torch.zeros(M, N, dtype=BF16, device="cuda"))
    y2, pre2 = vmb.vmb_linear_fwd(x, w, b, act=act, residual=None if res is None else off(res), y=out, want_pre=want_pre)
    assert y2.data_ptr() == out.data_ptr() and out.data_ptr() % 16 == 2
    close(out, want, K)
    assert not want_pre or torch.equal(pre2, pre)
    assert vmb.vmb_read_status(vmb.layer_workspace()) == vmb.VMB_OK


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("act,bias,residual,want_pre", EPILOGUES)
def test_eight_bits(vmb, M, K, N, act, bias, residual, want_pre):
    assert parts(vmb, M, 2 * K, N, True) > 1
    r = rand(M + 5 * K + N)
    (x, xs), (w, ws) = eight(r(M, 2 * K)), eight(r(N, 2 * K) / (2 * K) ** 0.5)
    b, res = r(N) if bias else None, r(M, N).to(BF16) if residual else None
    y, pre = vmb.vmb_linear_fwd(x, w, b, act=act, residual=res, x_scale=xs, weight_scale=ws, want_pre=want_pre)
    want, z = product(x, w, b, act, res, xs, ws)
    close(y, want, 2 * K)
    if want_pre:
        close(pre, z, 2 * K)


@pytest.mark.parametrize("M,K,N", [(64, 1000, 2048), (2048, 72, 264), (4096, 40, 33), (3000, 128, 136)])
def test_gradients(vmb, M, K, N):
    """dx contracts over N, dweight over M; odd N takes the kernel of any strides."""
    if N % 8 == 0:
        assert max(parts(vmb, M, N, K), parts(vmb, N, M, K)) > 1
    r = rand(M + K + 7 * N)
    x, w, dy = r(M, K).to(BF16), (r(N, K) / K ** 0.5).to(BF16), r(M, N).to(BF16)
    d = vmb.vmb_linear_bwd(x, w, dy, want_bias=True)
    dx, dw = dy.double() @ w.double(), dy.double().t() @ x.double()
    assert ref.rel(d["x"], dx) <= tol(N) and ref.rel(d["weight"], dw) <= tol(M)
    # element by element: dx sums N products of order 1 / sqrt(K), dweight M of order one, each sum off by 2^-20 of its terms at most
    assert ((d["x"].double() - dx).abs() <= 2.0 ** -8 * dx.abs() + N * 2.0 ** -20).all()
    assert ((d["weight"].double() - dw).abs() <= 2.0 ** -8 * dw.abs() + M * 2.0 ** -20).all()
