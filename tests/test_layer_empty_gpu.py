"""Gradients of empty problems: what has elements still is written, as the sum of nothing.  Through the C entry points, over outputs that hold something
else, and through Python."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def vmb():
    import paper_2412_16602_gb300 as vmb
    return vmb


def full(*shape, dtype=F32):
    return torch.full(shape, 7.0, device="cuda", dtype=dtype)


def stream():
    return torch.cuda.current_stream().cuda_stream


def test_convolution(vmb):
    dw, db, ws = full(40, 4), full(40), torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert vmb.lib.vmb_causal_conv_bwd(0, 0, 0, None, 0, 0, 0, 0, 0, dw.data_ptr(), db.data_ptr(), 0, 0, 5, 0, 40, 4, 1, 0, ws.data_ptr(), 256, stream()) == 0
    assert not dw.any() and not db.any()
    for offsets in (None, torch.zeros(1, dtype=torch.int32, device="cuda")):  # (no rows; one row of no tokens and no sequences)
        x = full(0, 5, 40) if offsets is None else full(1, 0, 40)
        d = vmb.vmb_causal_conv_bwd(x, full(40, 4), full(40), x, offsets=offsets)
        assert not d["weight"].any() and not d["bias"].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan(vmb, dtype):
    outs = [full(24, 16), full(24), full(24)]
    assert vmb.lib.vmb_token_scan_bwd(*[0] * 8, None, 0, 0, 0, 0, 0, 0, outs[0].data_ptr(), 0, 0, outs[1].data_ptr(), outs[2].data_ptr(), 0, 0, 0, 5, 0, 24, 16,
                                      1, int(dtype == BF16), 0, 0, stream()) == 0
    assert not any(t.any() for t in outs)
    dB, dC = full(2, 5, 16, dtype=dtype), full(2, 5, 16, dtype=dtype)  # (tokens of no channels)
    assert vmb.lib.vmb_token_scan_bwd(*[0] * 8, None, 0, 0, 0, 0, 0, 0, 0, dB.data_ptr(), dC.data_ptr(), 0, 0, 0, 0, 2, 5, 10, 0, 16, 1, int(dtype == BF16), 0,
                                      0, stream()) == 0
    assert not dB.any() and not dC.any()
    for B, T, D in ((0, 5, 24), (2, 5, 0)):
        x, Bm, A = full(B, T, D, dtype=dtype), full(B, T, 16, dtype=dtype), full(D, 16)
        rubbish = [full(2, 5, 16, dtype=dtype) for _ in range(8)]  # (what the outputs' memory holds)
        _, _, saved = vmb.vmb_token_scan_fwd(x, x, A, Bm, Bm, full(D), full(D), x, want_saved=True)
        del rubbish
        d = vmb.vmb_token_scan_bwd(x, x, A, Bm, Bm, full(D), full(D), x, x, saved)
        assert not any(t.any() for t in d.values())


def test_norm(vmb):
    dw = full(64)
    assert vmb.lib.vmb_rms_norm_bwd(0, 0, 0, 0, 0, 0, dw.data_ptr(), 0, 64, 0, 0, 0, stream()) == 0
    assert not dw.any()
    d = vmb.vmb_rms_norm_bwd(full(0, 64), full(64), full(0), full(0, 64))
    assert d["x"].shape == (0, 64) and not d["weight"].any()


def test_product(vmb):
    dw, db, dx = full(40, 24, dtype=BF16), full(40), full(6, 24, dtype=BF16)
    assert vmb.lib.vmb_linear_bwd(0, 24, 0, 0, 0, 0, dw.data_ptr(), db.data_ptr(), 0, 24, 40, 0, 0, 0, stream()) == 0
    assert not dw.any() and not db.any()
    assert vmb.lib.vmb_linear_bwd(0, 24, 0, 0, 0, dx.data_ptr(), 0, 0, 6, 24, 0, 0, 0, 0, stream()) == 0
    assert not dx.any()
    for M, N in ((0, 40), (6, 0)):
        d = vmb.vmb_linear_bwd(full(M, 24, dtype=BF16), full(N, 24, dtype=BF16), full(M, N, dtype=BF16), want_bias=True)
        assert d["x"].shape == (M, 24) and not any(t.any() for t in d.values())
