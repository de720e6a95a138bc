"""Packed sequences in a token buffer with rows that none of them holds: these are zero in the output and in every gradient,
whatever was in the outputs' and the workspace's memory; all others have the bits of a
buffer without them (the same plan; other addresses)."""
import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def run(x, do, offsets, max_len, ws):
    import paper_2412_16602_gb300 as vmb
    new = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    q, k, v, g, beta = x
    N, total, (Hk, Dk), (Hv, Dv) = offsets.numel() - 1, q.shape[1], q.shape[2:], v.shape[2:]
    dt, s = 0 if q.dtype == torch.float32 else 1, torch.cuda.current_stream().cuda_stream
    ws.fill_(255)
    ws[:256] = 0
    saved = torch.full((vmb.vmb_delta_rule_saved_bytes(N, max_len, total, True, Hv, Dk, Dv, q.dtype),), 255, dtype=torch.uint8, device="cuda")
    o, d = new(v), [new(t) for t in x]
    p = lambda *ts: [t.data_ptr() for t in ts]  # noqa: E731
    sizes = (N, max_len, total, Hk, Hv, Dk, Dv, Dk ** -0.5, dt, ws.data_ptr(), ws.numel(), s)
    assert vmb.lib.vmb_delta_rule_fwd(*p(*x), None, None, offsets.data_ptr(), o.data_ptr(), None, saved.data_ptr(), *sizes) == vmb.VMB_OK
    assert vmb.lib.vmb_delta_rule_bwd(*p(q, k, g, beta), None, offsets.data_ptr(), do.data_ptr(), None, saved.data_ptr(), *p(*d), None,
                                      *sizes) == vmb.VMB_OK
    return [o, *d], vmb.vmb_read_status(ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 2, 64, 48), (1, 3, 100, 40), (2, 2, 9, 5), (1, 2, 127, 131)])
@pytest.mark.parametrize("before,behind", [(0, 37), (5, 0), (70, 2000)])
def test_rows_of_no_sequence(size, before, behind, dtype):
    import paper_2412_16602_gb300 as vmb
    Hk, Hv, Dk, Dv = size
    lens = (65, 0, 130, 3)
    held = sum(lens)
    ws = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    x = [t.cuda() for t in ref.inputs(1, held, Hk, Hv, Dk, Dv, 71, TYPES[dtype])]
    do = torch.randn(1, held, Hv, Dv, device="cuda").to(TYPES[dtype])
    at = torch.tensor([0, 65, 65, 195, 198], dtype=torch.int32, device="cuda")
    want, status = run(x, do, at, max(lens), ws)
    assert status == vmb.VMB_OK

    def padded(t):
        fill = lambda n: torch.full((1, n, *t.shape[2:]), float("nan"), dtype=t.dtype, device="cuda")  # noqa: E731
        return torch.cat([fill(before), t, fill(behind)], 1).contiguous()

    got, status = run([padded(t) for t in x], padded(do), at + before, max(lens), ws)
    assert status == vmb.VMB_OK
    for a, b in zip(got, want):
        assert torch.equal(a[:, before:before + held], b)
        assert (a[:, :before] == 0).all() and (a[:, before + held:] == 0).all()


def test_rows_beyond_a_bound_and_odd_addresses():
    """A sequence longer than the bound is cut: its other rows are zero too.  Rows of two bytes and of odd numbers of them."""
    import paper_2412_16602_gb300 as vmb
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for Dk, Dv in ((3, 1), (16, 7)):
        x = [t.cuda() for t in ref.inputs(1, 120, 1, 1, Dk, Dv, 73, torch.bfloat16)]
        x = [torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape) for t in x]
        got, status = run(x, x[2].clone(), torch.tensor([0, 50, 110], dtype=torch.int32, device="cuda"), 40, ws)
        assert status == vmb.VMB_ERR_BOUNDS
        for t in got:
            assert torch.isfinite(t).all()
            assert (t[:, 40:50] == 0).all() and (t[:, 90:] == 0).all() and (t[:, :40] != 0).any() and (t[:, 50:90] != 0).any()


def test_no_sequences_at_all():
    import paper_2412_16602_gb300 as vmb
    x = [t.cuda() for t in ref.inputs(1, 30, 1, 2, 16, 8, 72)]
    kw = dict(offsets=torch.zeros(1, dtype=torch.int32, device="cuda"), max_len=0)
    for t in [torch.full((1, 30, 2, 16), float("nan"), device="cuda") for _ in range(8)]:
        del t
    o, S, saved = vmb.vmb_delta_rule_fwd(*x, want_state=True, want_saved=True, **kw)
    d = vmb.vmb_delta_rule_bwd(*x, torch.ones_like(x[2]), saved, **kw)
    assert S.shape[0] == 0 and (o == 0).all() and all((t == 0).all() for t in d.values())
