"""The norm's weight wherever a slice of a flat buffer of parameters lies: any number of floats past a multiple of 32 bytes gives the
bits of the same weight at a multiple of 512."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,C", [(3, 64), (40, 1536), (5, 8192)])
@pytest.mark.parametrize("floats", [4, 8, 12, 20])  # (others than multiples of four are taken one by one)
def test_weight_past_a_multiple_of_32_bytes(dtype, rows, C, floats):
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator(device="cuda").manual_seed(C + floats)
    x, dy = (torch.randn(rows, C, device="cuda", generator=g).to(dtype) for _ in range(2))
    flat = torch.randn(floats + C, device="cuda", generator=g)
    w, plain = flat[floats:], flat[floats:].clone()
    assert w.data_ptr() % 32 == 4 * floats % 32 and plain.data_ptr() % 512 == 0
    for bits8 in (False, True):
        got, want = (vmb.vmb_rms_norm_fwd(x, t, bits8=bits8, want_stats=True) for t in (w, plain))
        assert all(a is b is None or torch.equal(a.float(), b.float()) for a, b in zip(got, want))
    got, want = (vmb.vmb_rms_norm_bwd(x, t, want[3], dy) for t in (w, plain))
    assert torch.equal(got["x"], want["x"]) and torch.equal(got["weight"], want["weight"])
