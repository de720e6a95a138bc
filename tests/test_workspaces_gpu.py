"""Calls with their default workspaces on several streams, in several threads and in captured graphs: every result has the
bits of the same call alone."""
import threading

import pytest
import torch

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture
def calls(monkeypatch):
    """(call(stream), its result alone) of a chain in segments, its gradients, and norms in two passes over memory (what is
    larger than a cluster) and in clusters, with fresh default workspaces behind them."""
    import paper_2412_16602_gb300 as vmb
    torch.manual_seed(3)
    d = [t.cuda() for t in ref.inputs(1, 700, 1, 2, 64, 64, 51)]
    do = torch.randn(1, 700, 2, 64, device="cuda")
    big, small = torch.randn(3, 60, 70, 66, device="cuda") + 2, torch.randn(4, 30, 30, 64, device="cuda")
    w, b = torch.rand(66, device="cuda") + 0.5, torch.randn(66, device="cuda")

    def delta(stream=None):
        o, S, saved = vmb.vmb_delta_rule_fwd(*d, want_state=True, want_saved=True, stream=stream)
        return [o, S, *vmb.vmb_delta_rule_bwd(*d, do, saved, stream=stream).values()]

    def norm(x, w, b, G):
        def run(stream=None):
            y, stats = vmb.vmb_group_norm_fwd(x, w, b, G, act="gelu", want_stats=True, stream=stream)
            return [y, stats, *(t for t in vmb.vmb_group_norm_bwd(x, w, b, stats, x, G, act="gelu", stream=stream).values() if t is not None)]
        return run

    fs = [delta, norm(big, w, b, 3), norm(small, None, None, 8)]
    alone = [[t.clone() for t in f()] for f in fs]
    torch.cuda.synchronize()
    for name in ("_delta_ws", "_norm_ws"):
        monkeypatch.setattr(vmb.vmb, name, vmb.vmb.Workspace())
    return list(zip(fs, alone))


def same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


def test_first_use_on_a_stream_that_is_not_the_current_one(calls):
    """The memory that the workspace gets holds something else, and the current stream is busy for some time."""
    rubbish = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 20, 1 << 22, 1 << 24)]
    del rubbish
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    got = [f(s) for f, _ in calls]
    s.synchronize()
    assert all(same(g, want) for g, (_, want) in zip(got, calls))
    torch.cuda.synchronize()


def test_streams_side_by_side(calls):
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [(f(s), want) for _ in range(10) for s in streams for f, want in calls]
    torch.cuda.synchronize()
    assert all(same(g, want) for g, want in got)


def test_threads_on_one_stream(calls):
    wrong = []

    def work():
        for _ in range(20):
            for f, want in calls:
                got = f()
                torch.cuda.current_stream().synchronize()
                if not same(got, want):
                    wrong.append(f)

    threads = [threading.Thread(target=work) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_growth_while_the_stream_is_busy(calls):
    import paper_2412_16602_gb300 as vmb
    s = torch.cuda.Stream()
    x = [t.cuda() for t in ref.inputs(1, 300, 1, 1, 32, 32, 52)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        first = vmb.vmb_delta_rule_fwd(*x)[0]
    got = [f(s) for f, _ in calls]
    s.synchronize()
    assert all(same(g, want) for g, (_, want) in zip(got, calls))
    assert torch.equal(first, vmb.vmb_delta_rule_fwd(*x)[0])


def test_captured_calls_beside_others(calls):
    """A graph's first replay, replays in a row, and calls outside between them."""
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        inside = [f() for f, _ in calls]
    for _ in range(3):
        for t in (t for ts in inside for t in ts):
            t.zero_()
        graph.replay()
        outside = [f(s) for f, _ in calls]
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(g, want) for g, (_, want) in zip(inside, calls))
        assert all(same(g, want) for g, (_, want) in zip(outside, calls))


def test_status_of_the_scans_workspaces():
    """The error word is read wherever the thread's scans ran."""
    import paper_2412_16602_gb300 as vmb
    s = torch.cuda.Stream()
    ws = vmb.default_workspace(stream=s)
    assert ws.data_ptr() != vmb.default_workspace().data_ptr()
    assert vmb.vmb_read_status() == vmb.VMB_OK
    ws[12:16] = torch.tensor([2, 0, 0, 0], dtype=torch.uint8, device="cuda")  # the header's error word: an index check
    assert vmb.vmb_read_status() == vmb.VMB_ERR_BOUNDS and vmb.vmb_read_status() == vmb.VMB_OK
