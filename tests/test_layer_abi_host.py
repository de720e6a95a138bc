"""The entry points of a layer around the scan over tokens without a GPU: sizes of workspaces, and every refusal before the
device is touched."""
import ctypes

import pytest

FAKE, OUT, WS, S = 0x10000, 0x20000, 0x100000, 0  # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def vmb():
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    return vmb


def strides(*v):
    return (ctypes.c_int64 * len(v))(*v)


def test_conv_refuses(vmb):
    def fwd(x=FAKE, w=FAKE, b=0, st=None, init=0, offs=0, y=OUT, final=0, B=1, T=8, total=None, C=16, W=4, act=1, dtype=0):
        return vmb.lib.vmb_causal_conv_fwd(x, w, b, st, init, offs, y, final, B, T, B * T if total is None else total, C, W, act, dtype, S)

    assert fwd(B=-1) == 1 and fwd(T=-1) == 1 and fwd(C=-1) == 1 and fwd(W=0) == 1 and fwd(W=5) == 3 and fwd(act=2) == 1 and fwd(dtype=4) == 1
    assert fwd(total=9) == 1 and fwd(x=0) == 1 and fwd(w=0) == 1 and fwd(y=0) == 1 and fwd(y=FAKE) == 1
    assert fwd(init=FAKE, final=FAKE) == 1 and fwd(x=FAKE + 2) == 2 and fwd(w=FAKE + 2) == 2 and fwd(b=FAKE + 1) == 2 and fwd(offs=FAKE + 2, total=8) == 2
    assert fwd(x=FAKE + 1, dtype=1) == 2 and fwd(st=strides(-1, 16)) == 1 and fwd(st=strides(0, -16)) == 1
    assert fwd(B=1 << 30, T=1 << 30, total=1 << 60, C=1 << 20) == 1 and fwd(B=1 << 20, T=1 << 12) == 3
    assert fwd(C=0, x=0, w=0, y=0) == 0 and fwd(B=0, x=0, w=0, y=0) == 0

    def bwd(n=1 << 30, ws=WS, dtype=0, **kw):
        a = dict(x=FAKE, w=FAKE, b=0, st=None, init=0, offs=0, dy=FAKE, dlast=0, dx=OUT, dw=OUT, db=OUT, dinit=0)
        a.update(kw)
        return vmb.lib.vmb_causal_conv_bwd(*a.values(), 1, 8, 8, 16, 4, 1, dtype, ws, n, S)

    for name in ("x", "w", "dy", "dx", "dw"):
        assert bwd(**{name: 0}) == 1, name
        assert bwd(**{name: FAKE + 2}) == 2, name
    assert bwd(dx=FAKE) == 1 and bwd(dinit=OUT, dlast=OUT) == 1 and bwd(db=OUT + 2) == 2 and bwd(ws=0) == 4 and bwd(ws=WS + 8) == 2 and bwd(n=64) == 4

    def step(x=FAKE, state=OUT * 2, slots=0, y=OUT, B=2, T=1, W=4, pool=2):
        return vmb.lib.vmb_causal_conv_step(x, FAKE, 0, None, state, slots, y, B, T, 16, W, pool, 1, 0, S)

    assert step(pool=1) == 1 and step(pool=-1) == 1 and step(state=0) == 1 and step(y=0) == 1 and step(y=FAKE) == 1 and step(state=OUT) == 1
    assert step(W=5) == 3 and step(slots=OUT + 1) == 2 and step(state=OUT + 2) == 2 and step(T=0) == 0 and step(B=0) == 0


def test_scan_refuses(vmb):
    order = ("x", "delta", "A", "Bm", "Cm", "skip", "bias", "z")

    def fwd(st=None, init=0, offs=0, y=OUT, final=0, saved=0, B=1, T=8, total=None, D=16, N=16, flags=1, dtype=0, ws=WS, n=1 << 30, **kw):
        ins = dict.fromkeys(order, FAKE)
        ins.update(kw)
        return vmb.lib.vmb_token_scan_fwd(*ins.values(), st, init, offs, y, final, saved, B, T, B * T if total is None else total, D, N, flags, dtype,
                                          ws, n, S)

    for name in ("x", "delta", "A", "Bm", "Cm"):
        assert fwd(**{name: 0}) == 1, name
    for name in order:
        assert fwd(**{name: FAKE + 2}) == 2, name
    assert fwd(N=0) == 1 and fwd(N=17) == 3 and fwd(flags=2) == 1 and fwd(dtype=2) == 1 and fwd(total=7) == 1 and fwd(T=-1) == 1
    assert fwd(y=0) == 1 and fwd(y=FAKE) == 1 and fwd(y=OUT + 2) == 2 and fwd(saved=OUT + 8) == 2 and fwd(init=OUT, final=OUT) == 1
    assert fwd(st=strides(*([16] * 9), -1)) == 1 and fwd(ws=0) == 4 and fwd(ws=WS + 32) == 2 and fwd(n=100) == 4
    assert fwd(B=1 << 20, T=1 << 12) == 3 and fwd(D=0, A=0) == 0 and fwd(B=0, ws=0) == 0

    outs = ("dx", "ddelta", "dA", "dB", "dC", "dD", "dbias", "dz")

    def bwd(offs=0, dy=FAKE, dlast=0, saved=FAKE, dinit=0, n=1 << 30, **kw):
        ins, o = dict.fromkeys(order, FAKE), dict.fromkeys(outs, OUT)
        ins.update({k: v for k, v in kw.items() if k in order})
        o.update({k: v for k, v in kw.items() if k in outs})
        return vmb.lib.vmb_token_scan_bwd(*ins.values(), None, offs, dy, dlast, saved, *o.values(), dinit, 1, 8, 8, 16, 16, 1, 0, WS, n, S)

    for name in ("x", "delta", "A", "Bm", "Cm", "dx", "ddelta", "dA", "dB", "dC", "dz", "dy", "saved"):
        assert bwd(**{name: 0}) == 1, name
    for name in ("dx", "ddelta", "dB", "dC", "dz"):
        assert bwd(**{name: FAKE}) == 1, name
        assert bwd(**{name: OUT + 2}) == 2, name
    assert bwd(dinit=OUT, dlast=OUT) == 1 and bwd(saved=FAKE + 8) == 2 and bwd(n=64) == 4

    def step(state=OUT * 2, slots=0, y=OUT, B=2, T=1, N=16, pool=2, A=FAKE):
        return vmb.lib.vmb_token_scan_step(FAKE, FAKE, A, FAKE, FAKE, 0, 0, 0, None, state, slots, y, B, T, 16, N, pool, 1, 0, S)

    assert step(pool=1) == 1 and step(pool=-1) == 1 and step(state=0) == 1 and step(y=0) == 1 and step(y=FAKE) == 1 and step(A=0) == 1
    assert step(N=17) == 3 and step(slots=OUT + 1) == 2 and step(state=OUT + 2) == 2 and step(T=0) == 0 and step(B=0) == 0


def test_norm_refuses(vmb):
    def fwd(x=FAKE, res=0, w=0, y=OUT, total=0, scale=0, rstd=0, rows=4, C=64, eps=1e-6, dtype=0):
        return vmb.lib.vmb_rms_norm_fwd(x, res, w, y, total, scale, rstd, rows, C, eps, dtype, S)

    assert fwd(rows=-1) == 1 and fwd(C=-1) == 1 and fwd(C=8193) == 3 and fwd(rows=1 << 31) == 3 and fwd(eps=-1.0) == 1 and fwd(eps=float("nan")) == 1
    assert fwd(x=0) == 1 and fwd(y=0) == 1 and fwd(y=FAKE) == 1 and fwd(res=FAKE) == 1 and fwd(res=FAKE, total=OUT) == 1 and fwd(dtype=2) == 1
    assert fwd(res=FAKE, total=FAKE) == 1
    assert fwd(x=FAKE + 2) == 2 and fwd(y=OUT + 2) == 2 and fwd(w=FAKE + 2) == 2 and fwd(rstd=FAKE + 2) == 2
    assert fwd(rows=0, x=0, y=0) == 0 and fwd(C=0, x=0, y=0) == 0

    def bwd(x=FAKE, w=0, rstd=FAKE, dy=FAKE, dsum=0, dx=OUT, dw=0, ws=WS, n=1 << 30):
        return vmb.lib.vmb_rms_norm_bwd(x, w, rstd, dy, dsum, dx, dw, 4, 64, 0, ws, n, S)

    assert bwd(x=0) == 1 and bwd(rstd=0) == 1 and bwd(dy=0) == 1 and bwd(dx=0) == 1 and bwd(dx=FAKE) == 1 and bwd(dsum=OUT) == 1
    assert bwd(dy=FAKE + 2) == 2 and bwd(dw=OUT + 2) == 2 and bwd(ws=0) == 4 and bwd(ws=WS + 4) == 2 and bwd(dw=OUT, n=64) == 4


def test_linear_refuses(vmb):
    def fwd(x=FAKE, x_t=64, w=FAKE, xs=0, ws_=0, b=0, res=0, y=OUT, pre=0, M=4, K=64, N=32, act=0, ws=WS, n=1 << 30):
        return vmb.lib.vmb_linear_fwd(x, x_t, w, xs, ws_, b, res, y, pre, M, K, N, act, ws, n, S)

    assert fwd(M=-1) == 1 and fwd(K=-1) == 1 and fwd(N=-1) == 1 and fwd(act=3) == 1 and fwd(x_t=-1) == 1 and fwd(xs=FAKE) == 1 and fwd(ws_=FAKE) == 1
    assert fwd(M=1 << 40, K=1 << 30) == 1 and fwd(M=1 << 31) == 3 and fwd(x_t=1 << 62) == 1
    assert fwd(x=0) == 1 and fwd(w=0) == 1 and fwd(y=0) == 1 and fwd(y=FAKE) == 1 and fwd(res=OUT) == 1 and fwd(pre=OUT) == 1 and fwd(pre=FAKE) == 1
    assert fwd(x=FAKE + 1) == 2 and fwd(y=OUT + 1) == 2 and fwd(b=FAKE + 2) == 2 and fwd(xs=FAKE + 2, ws_=FAKE) == 2
    assert fwd(ws=0) == 4 and fwd(ws=WS + 8) == 2 and fwd(n=64) == 4
    assert fwd(M=0, x=0, w=0, y=0) == 0 and fwd(N=0, x=0, w=0, y=0) == 0

    def bwd(x=FAKE, x_t=64, w=FAKE, pre=0, dy=FAKE, dx=OUT, dw=OUT * 2, db=0, act=0, ws=WS, n=1 << 30):
        return vmb.lib.vmb_linear_bwd(x, x_t, w, pre, dy, dx, dw, db, 4, 64, 32, act, ws, n, S)

    assert bwd(x=0) == 1 and bwd(w=0) == 1 and bwd(dy=0) == 1 and bwd(act=1) == 1 and bwd(dx=FAKE) == 1 and bwd(dw=OUT) == 1 and bwd(x_t=-1) == 1
    assert bwd(dy=FAKE + 1) == 2 and bwd(db=OUT + 2) == 2 and bwd(ws=0) == 4 and bwd(n=64) == 4 and bwd(act=1, pre=OUT) == 1


def test_sizes(vmb):
    ws = vmb.vmb_token_scan_workspace_bytes
    assert ws(1, 8, 9, False, 16, 16) == 0 and ws(1, 8, 8, False, 16, 17) == 0 and ws(0, 8, 0, False, 16, 16) == 256
    assert ws(2, 100, 200, False, 64, 16, True) > ws(2, 100, 200, False, 64, 16)
    saved = vmb.vmb_token_scan_saved_bytes  # the states before every 16 tokens
    assert saved(3, 65, 195, False, 8, 4) == 3 * 5 * 8 * 4 * 4 + 256
    assert saved(3, 0, 195, True, 8, 4) == (195 // 16 + 3) * 8 * 4 * 4 + 256
    assert vmb.vmb_causal_conv_workspace_bytes(1, 8, 9, False, 16, 4) == 0 and vmb.vmb_causal_conv_workspace_bytes(1, 8, 8, False, 16, 5) == 0
    assert vmb.vmb_rms_norm_workspace_bytes(4, 8193) == 0 and vmb.vmb_rms_norm_workspace_bytes(0, 64) == 256
    assert vmb.vmb_linear_workspace_bytes(-1, 8, 8) == 0 and vmb.vmb_linear_workspace_bytes(0, 8, 8) == 256
    assert vmb.vmb_linear_workspace_bytes(64, 8, 256, True) >= 64 * 256 * 2
