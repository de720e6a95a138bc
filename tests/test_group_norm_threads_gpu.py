"""Norms of wide maps in two threads: each launch has the shared memory that its own width needs."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_two_widths_at_once():
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(9)
    xs = [torch.randn(1, 4, C, device="cuda") for C in (16384, 6144)]
    want = [vmb.vmb_group_norm_fwd(x, None, None, 1)[0] for x in xs]
    torch.cuda.synchronize()
    start, errors = threading.Barrier(2), []

    def work(x, y):
        start.wait()
        try:
            for _ in range(5000):
                got = vmb.vmb_group_norm_fwd(x, None, None, 1)[0]
            assert torch.equal(got, y)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(xs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
