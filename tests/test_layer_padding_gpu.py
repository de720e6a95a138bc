"""Packed batches as a serving loop has them: a token buffer whose padding holds what is not a number, and a captured graph whose offsets change between
replays.  Outputs, states and gradients have the bits of the same call over clean padding, or made anew."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
T, C, N = 700, 72, 16


def make(dtype, n):
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    rows = dict(x=r(1, T, C).to(dtype), delta=r(1, T, C).to(dtype), B=r(1, T, N).to(dtype), C=r(1, T, N).to(dtype), z=r(1, T, C).to(dtype), dy=r(1, T, C).to(dtype))
    rest = dict(A=-4 * torch.rand(C, N, device="cuda", generator=g), skip=r(C), bias=r(C) - 2, w=r(C, 4), b=r(C), init=r(n, C, N), seen=r(n, 3, C).to(dtype),
                dlast=r(n, C, N), dseen=r(n, 3, C).to(dtype))
    return rows, rest


def run(rows, k, offsets):
    import paper_2412_16602_gb300 as vmb
    y, last = vmb.vmb_causal_conv_fwd(rows["x"], k["w"], k["b"], initial_state=k["seen"], offsets=offsets, want_state=True)
    d = vmb.vmb_causal_conv_bwd(rows["x"], k["w"], k["b"], rows["dy"], initial_state=k["seen"], dfinal_state=k["dseen"], offsets=offsets, want_initial=True)
    ins = [rows["x"], rows["delta"], k["A"], rows["B"], rows["C"], k["skip"], k["bias"], rows["z"]]
    o, h, saved = vmb.vmb_token_scan_fwd(*ins, initial_state=k["init"], offsets=offsets, want_state=True, want_saved=True)
    e = vmb.vmb_token_scan_bwd(*ins, rows["dy"], saved, dfinal_state=k["dlast"], offsets=offsets, want_initial=True)
    return {"y": y, "last": last, "o": o, "h": h, **{"conv " + n: t for n, t in d.items()}, **{"scan " + n: t for n, t in e.items()}}


def same(got, want):
    for n in want:
        assert torch.equal(got[n], want[n]), n


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("at", [[0, 100, 100, 350, 353], [61, 62, 300, 640], [0, 0, 699], [350, 350, 350]])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_padding_that_is_not_a_number(dtype, at, what):
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    rows, k = make(dtype, len(at) - 1)
    want = run(rows, k, offsets)
    dirty = {n: t.clone() for n, t in rows.items()}
    for t in dirty.values():
        t[:, :at[0]], t[:, at[-1]:] = what, what
    same(run(dirty, k, offsets), want)
    assert all(t.isfinite().all() for t in want.values())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_offsets_that_change_between_replays(dtype):
    layouts = [[0, 100, 100, 350, 353], [61, 62, 300, 640, 700], [0, 0, 0, 0, 700], [5, 5, 5, 5, 5], [0, 697, 698, 699, 700]]
    rows, k = make(dtype, 4)
    offsets = torch.tensor(layouts[0], dtype=torch.int32, device="cuda")
    run(rows, k, offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(rows, k, offsets)
    for at in (*layouts, layouts[0]):
        now = torch.tensor(at, dtype=torch.int32, device="cuda")
        offsets.copy_(now)
        graph.replay()
        same(got, run(rows, k, now))
