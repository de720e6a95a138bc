"""The short causal convolution at the sizes that its loops are for, against its definition in 64 bits as whole tensors: runs of 8 to 32 tokens, several runs a
thread in the gradients, packed batches whose sequences are found by a warp.

Tolerances: outputs as in the tests of small sizes.  The filter's gradients sum up to 80000 terms of random sign in chains of at most 200 fp32 additions (a
thread's, then the join of the threads'); no partial sum exceeds the whole's size in the norm by more than a factor of 2, and the roundings, 2^-24 each, are
independent: 2 sqrt(200) 2^-24 < 2^-19, the terms' own 2^-19 beside it.  2^-14 leaves room for chains of one sign; one token left out would be
1 / sqrt(80000) > 2^-9."""
import pytest
import torch

from tests import layer_reference as ref
from tests.test_causal_conv_gpu import BF16, F32, OUT, SUM, make

pytestmark = pytest.mark.gpu


def conv(x, w, b, initial, spans, act):
    """(y, final states) of sequences [(batch row, first token, one past the last)], tokens of no sequence zero; in 64 bits."""
    W, y, last = w.shape[1], torch.zeros_like(x), []
    rows = []
    for i, (row, t0, t1) in enumerate(spans):
        seen = torch.cat([initial[i], x[row, t0:t1]])
        z = sum(seen[j:j + t1 - t0] * w[:, j] for j in range(W)) + b
        rows.append((row, t0, t1, z * torch.sigmoid(z) if act == "silu" else z))
        last.append(seen[t1 - t0:])
    y = torch.cat([torch.cat([torch.zeros(t0 - (rows[i - 1][2] if i and rows[i - 1][0] == row else 0), x.shape[2], dtype=x.dtype, device=x.device), o])
                   for i, (row, t0, t1, o) in enumerate(rows)])
    return torch.cat([y, x.new_zeros(x.shape[0] * x.shape[1] - len(y), x.shape[2])]).view(x.shape), torch.stack(last)


def check(vmb, x, w, b, init, dy, dlast, spans, offsets, act):
    y, last = vmb.vmb_causal_conv_fwd(x, w, b, act=act, initial_state=init, offsets=offsets, want_state=True)
    leaves = [t.double().requires_grad_() for t in (x, w, b, init)]
    yr, lr = conv(*leaves, spans, act)
    assert ref.rel(y, yr.detach()) <= OUT[x.dtype] and torch.equal(last, lr.detach().to(x.dtype))
    # no element off by more than the sums of a window allow: five terms of order one, 2^-21 of them each, and the rounding to the storage type
    assert ((y.double() - yr.detach()).abs() <= ref.HALF[x.dtype] * yr.detach().abs() + 2.0 ** -16).all()
    want = torch.autograd.grad((yr * dy.double()).sum() + (lr * dlast.double()).sum(), leaves)
    del yr, lr, leaves
    got = vmb.vmb_causal_conv_bwd(x, w, b, dy, act=act, initial_state=init, dfinal_state=dlast, offsets=offsets, want_initial=True)
    assert ref.rel(got["x"], want[0]) <= OUT[x.dtype] and ref.rel(got["initial_state"], want[3]) <= OUT[x.dtype]
    assert ((got["x"].double() - want[0]).abs() <= ref.HALF[x.dtype] * want[0].abs() + 2.0 ** -15).all()
    assert ref.rel(got["weight"], want[1]) <= SUM and ref.rel(got["bias"], want[2]) <= SUM


@pytest.mark.parametrize("B,T,C,W,act,dtype", [(1, 80000, 512, 4, "silu", F32), (1, 80000, 512, 4, "silu", BF16), (8, 3136, 768, 3, "silu", F32),
                                               (3, 27001, 520, 4, "none", BF16), (2, 40001, 129, 2, "silu", F32), (5, 9999, 1536, 4, "silu", BF16),
                                               (1, 50000, 64, 1, "silu", BF16)])
def test_dense(B, T, C, W, act, dtype):
    import paper_2412_16602_gb300 as vmb
    x, w, b, init, dy, dlast = make(11, B, T, C, W, dtype)
    check(vmb, x, w, b, init, dy, dlast, [(i, 0, T) for i in range(B)], None, act)


@pytest.mark.parametrize("C,W,dtype,most", [(512, 4, F32, 1400), (512, 4, BF16, 1400), (1536, 4, BF16, 900), (516, 3, BF16, 300), (1030, 2, F32, 60), (61, 4, F32, 2500)])
@pytest.mark.parametrize("lead,tail", [(0, 0), (37, 300)])
def test_packed(C, W, dtype, most, lead, tail):
    import paper_2412_16602_gb300 as vmb
    g = torch.Generator().manual_seed(C)
    lens = [int(n) for n in torch.randint(0, most, (45,), generator=g)]
    for i, n in ((0, 0), (7, 0), (8, 0), (9, 1), (20, 2), (21, 3), (44, 0)):
        lens[i] = n
    at = [lead]
    for n in lens:
        at.append(at[-1] + n)
    x, w, b, init, dy, dlast = make(12, 1, at[-1] + tail, C, W, dtype, n=45)
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    check(vmb, x, w, b, init, dy, dlast, [(0, at[i], at[i + 1]) for i in range(45)], offsets, "silu")
