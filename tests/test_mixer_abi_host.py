"""The token mixer's entry points without a GPU: sizes of workspaces, and every refusal before the device is touched."""
import ctypes

import pytest

FAKE, WS, S = 0x10000, 0x100000, 0  # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def vmb():
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    return vmb


def fwd(vmb, B=1, T=8, total=None, Hk=2, Hv=2, Dk=16, Dv=16, dtype=0, ptrs=None, strides=None, init=0, offsets=0, o=FAKE * 2,
        final=0, saved=0, ws=WS, n=1 << 30):
    p = [FAKE] * 5 if ptrs is None else ptrs
    return vmb.lib.vmb_delta_rule_fwd(*p, strides, init, offsets, o, final, saved, B, T, B * T if total is None else total, Hk, Hv, Dk,
                                      Dv, 0.25, dtype, ws, n, S)


def test_delta_forward_refuses(vmb):
    ok = vmb.VMB_OK
    assert fwd(vmb, B=-1) == 1 and fwd(vmb, T=-1) == 1 and fwd(vmb, Hk=3) == 1 and fwd(vmb, dtype=5) == 1
    assert fwd(vmb, total=9) == 1                                   # not B * T
    assert fwd(vmb, Dk=129) == 3 and fwd(vmb, B=1 << 20, T=64, Hv=64, Hk=64) == 3
    assert fwd(vmb, B=1 << 30, T=1 << 30, total=1 << 60, Dk=128) == 1  # beyond int64
    for i in range(5):
        assert fwd(vmb, ptrs=[0 if j == i else FAKE for j in range(5)]) == 1
        assert fwd(vmb, ptrs=[FAKE + 2 if j == i else FAKE for j in range(5)]) == 2
    assert fwd(vmb, o=0) == 1 and fwd(vmb, o=FAKE) == 1 and fwd(vmb, o=FAKE * 2 + 2) == 2
    assert fwd(vmb, init=FAKE, final=FAKE) == 1 and fwd(vmb, init=FAKE + 2) == 2 and fwd(vmb, saved=FAKE + 8) == 2
    assert fwd(vmb, strides=(ctypes.c_int64 * 6)(0, -1, 0, 0, 0, 0)) == 1
    assert fwd(vmb, ws=0) == 4 and fwd(vmb, ws=WS + 16) == 2 and fwd(vmb, n=64) == 4
    assert fwd(vmb, B=0, ptrs=[0] * 5, o=0, ws=0) == ok and fwd(vmb, Hv=0, Hk=0, ptrs=[0] * 5, o=0, ws=0) == ok


def test_delta_backward_and_step_refuse(vmb):
    def bwd(skip=None, dtype=0, n=1 << 30, **kw):
        a = dict(q=FAKE, k=FAKE, g=FAKE, beta=FAKE, strides=None, offsets=0, do=FAKE, dfinal=0, saved=FAKE, dq=FAKE, dk=FAKE, dv=FAKE,
                 dg=FAKE, dbeta=FAKE, dinit=0)
        a.update(kw)
        if skip:
            a[skip] = 0
        return vmb.lib.vmb_delta_rule_bwd(*a.values(), 1, 8, 8, 2, 2, 16, 16, 0.25, dtype, WS, n, S)

    for name in ("q", "k", "g", "beta", "do", "saved", "dq", "dk", "dv", "dg", "dbeta"):
        assert bwd(name) == 1, name
        assert bwd(**{name: FAKE + 2}) == 2, name
    assert bwd(dtype=3) == 1 and bwd(n=100) == 4 and bwd(dinit=FAKE, dfinal=FAKE) == 1

    def step(B=2, T=1, pool=2, Dk=16, ptrs=None, state=FAKE, slots=0, o=FAKE):
        return vmb.lib.vmb_delta_rule_step(*(ptrs or [FAKE] * 5), None, state, slots, o, B, T, 2, 2, Dk, 16, pool, 0.25, 0, S)

    assert step(pool=1) == 1 and step(pool=-1) == 1 and step(state=0) == 1 and step(o=0) == 1 and step(Dk=200) == 3
    assert step(state=FAKE + 2) == 2 and step(slots=FAKE + 1) == 2 and step(ptrs=[FAKE] * 4 + [0]) == 1
    assert step(B=0, ptrs=[0] * 5, state=0, o=0) == 0 and step(T=0, ptrs=[0] * 5, state=0, o=0) == 0


def test_delta_sizes(vmb):
    ws = vmb.vmb_delta_rule_workspace_bytes
    assert ws(1, 8, 9, False, 1, 1, 16, 16) == 0 and ws(1, 8, 8, False, 2, 3, 16, 16) == 0 and ws(0, 8, 0, False, 1, 1, 16, 16) == 256
    # gradients need dS and dX; in fp32 with Dk > 64 shared heads leave their dq and dk to be summed
    assert ws(64, 64, 4096, False, 4, 4, 64, 64, True) > ws(64, 64, 4096, False, 4, 4, 64, 64)
    assert ws(64, 64, 4096, False, 2, 4, 128, 64, True) > ws(64, 64, 4096, False, 4, 4, 128, 64, True)
    saved = vmb.vmb_delta_rule_saved_bytes
    # chunk states [2 chunks][Hv][Dv][Dk] and residuals [tokens][Hv][Dv]
    assert saved(1, 65, 65, False, 2, 64, 32) == 2 * 2 * 64 * 32 * 4 + 65 * 2 * 32 * 4
    assert saved(3, 64, 130, True, 1, 64, 64) == (130 // 64 + 3) * 64 * 64 * 4 + 130 * 64 * 4


def test_rotary_refuses(vmb):
    def rot(q=FAKE, k=FAKE, freq=FAKE, pos=0, qo=FAKE, ko=FAKE, B=1, T=6, Hq=1, Hk=1, D=16, pairs=(4, 2), grid=(2, 3), strides=None,
            flags=0, dtype=0, axes=None):
        c = lambda v: None if v is None else (ctypes.c_int * max(1, len(v)))(*v)  # noqa: E731
        return vmb.lib.vmb_rotary_fwd(q, k, freq, pos, qo, ko, B, T, Hq, Hk, D, len(pairs) if axes is None else axes, c(pairs), c(grid),
                                      strides, flags, dtype, S)

    assert rot(B=-1) == 1 and rot(dtype=2) == 1 and rot(flags=4) == 1 and rot(axes=0) == 1 and rot(pairs=(1,) * 5, grid=(1,) * 5) == 1
    assert rot(pairs=(5, 4)) == 1 and rot(pairs=(0, 0)) == 1 and rot(pairs=(-1, 3)) == 1     # 2P > D, no pairs, negative
    assert rot(grid=(2, 2)) == 1 and rot(grid=None) == 1 and rot(grid=(-2, -3)) == 1         # cells are not T
    assert rot(q=0) == 1 and rot(k=0) == 1 and rot(freq=0) == 1 and rot(qo=0) == 1 and rot(ko=0) == 1
    assert rot(q=FAKE + 2) == 2 and rot(ko=FAKE + 1) == 2 and rot(pos=FAKE + 2) == 2
    assert rot(strides=(ctypes.c_int64 * 4)(-1, 0, 0, 0)) == 1
    assert rot(strides=(ctypes.c_int64 * 4)(200, 20, 96, 16)) == 1                           # in place with strided rows
    assert rot(D=1 << 20, pairs=(5000, 0)) == 3
    assert rot(B=0, q=0, k=0, qo=0, ko=0) == 0


def test_norm_refuses(vmb):
    def norm(x=FAKE, y=FAKE * 2, w=0, b=0, stats=0, B=2, L=5, C=12, G=3, eps=1e-5, act=1, dtype=0, ws=WS, n=1 << 30):
        return vmb.lib.vmb_group_norm_fwd(x, w, b, y, stats, B, L, C, G, eps, act, dtype, ws, n, S)

    assert norm(B=-1) == 1 and norm(G=5) == 1 and norm(G=0) == 1 and norm(act=3) == 1 and norm(dtype=9) == 1 and norm(eps=-1.0) == 1
    assert norm(eps=float("nan")) == 1 and norm(x=0) == 1 and norm(y=0) == 1 and norm(y=FAKE) == 1 and norm(C=16386) == 3
    assert norm(x=FAKE + 2) == 2 and norm(w=FAKE + 2) == 2 and norm(stats=FAKE + 4) == 2
    assert norm(ws=0) == 4 and norm(ws=WS + 8) == 2 and norm(n=256) == 4
    assert norm(B=0, x=0, y=0, ws=0) == 0 and norm(L=0, x=0, y=0, ws=0) == 0

    def bwd(x=FAKE, stats=FAKE, dy=FAKE * 2, dx=FAKE * 3):
        return vmb.lib.vmb_group_norm_bwd(x, 0, 0, stats, dy, dx, 0, 0, 2, 5, 12, 3, 1, 0, WS, 64, S)

    assert bwd(x=0) == 1 and bwd(stats=0) == 1 and bwd(dy=0) == 1 and bwd(dx=0) == 1 and bwd(dx=FAKE) == 1 and bwd(dx=FAKE * 2) == 1
    assert bwd() == 4
    assert vmb.vmb_group_norm_workspace_bytes(2, 5, 12, 5) == 0 and vmb.vmb_group_norm_workspace_bytes(0, 5, 12, 3) == 256
