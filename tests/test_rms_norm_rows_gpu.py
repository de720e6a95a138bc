"""Gradients of the norm for more rows than its blocks take at once, against the definition in 64 bits: the next row's values ahead, and sums over several rows of a
thread.  Tolerances: dx as in the tests of few rows; the weight's gradient sums up to 12000 terms of random sign in chains of some 100 additions: 2^-13 as there
(one row left out would be 1 / sqrt(12000) > 2^-7)."""
import pytest
import torch

from tests import layer_reference as ref
from tests.test_rms_norm_gpu import BF16, F32, make, norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,C,dtype", [(12000, 128, F32), (12000, 128, BF16), (3000, 8192, BF16), (3000, 8192, F32), (9001, 768, F32), (5003, 1536, BF16),
                                          (4001, 1001, BF16), (7000, 4096, F32), (2999, 8191, F32)])
@pytest.mark.parametrize("weight,dsum", [(True, True), (True, False), (False, True)])
def test_gradients(rows, C, dtype, weight, dsum):
    import paper_2412_16602_gb300 as vmb
    x, w, _, dy, ds = make(rows, C, dtype, 21)
    w, ds = w if weight else None, ds if dsum else None
    _, _, _, rstd = vmb.vmb_rms_norm_fwd(x, w, want_stats=True)
    got = vmb.vmb_rms_norm_bwd(x, w, rstd, dy, dsum=ds)
    leaves = [t.double().requires_grad_() for t in ((x, w) if weight else (x,))]
    y = norm(leaves[0], leaves[1] if weight else None)
    loss = (y * dy.double()).sum() + (0 if ds is None else (leaves[0] * ds.double()).sum())
    want = torch.autograd.grad(loss, leaves)
    terms = (rstd.double().unsqueeze(1) * dy.double() * (1.0 if w is None else w.double())).norm(dim=1)
    off = (got["x"].double() - want[0]).norm(dim=1)  # (row by row: a mistake in one is not lost among the others)
    assert (off <= 2.0 ** -17 * terms + (2.0 ** -18 + ref.HALF[dtype]) * want[0].norm(dim=1)).all()
    if weight:
        assert ref.rel(got["weight"], want[1]) <= 2.0 ** -13
