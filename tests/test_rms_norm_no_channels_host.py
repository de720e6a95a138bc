"""Rows of no channels have no mean: their statistics are refused instead of left as the memory was.  No GPU needed."""
import pytest
import torch

FAKE = 0x10000  # never dereferenced


@pytest.fixture(scope="module")
def vmb():
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    return vmb


def test_statistics_of_no_channels_are_refused(vmb):
    def fwd(rows, C, scale=0, rstd=0):
        return vmb.lib.vmb_rms_norm_fwd(0, 0, 0, 0, 0, scale, rstd, rows, C, 1e-6, 0, 0)

    assert fwd(5, 0, scale=FAKE) == vmb.VMB_ERR_INVALID_ARG and fwd(5, 0, rstd=FAKE) == vmb.VMB_ERR_INVALID_ARG
    assert fwd(5, 0) == vmb.VMB_OK and fwd(0, 0, FAKE, FAKE) == vmb.VMB_OK and fwd(0, 64, FAKE, FAKE) == vmb.VMB_OK


def test_rows_of_no_channels_are_counted(vmb, monkeypatch):
    monkeypatch.setattr(vmb.vmb, "_dev", lambda t, name: None)
    for shape, rows in (((5, 0), 5), ((2, 3, 0), 6), ((0,), 1), ((0, 0), 0), ((4, 8), 4)):
        assert vmb.vmb._rms_inputs(torch.empty(shape), None)[:2] == (rows, shape[-1])
