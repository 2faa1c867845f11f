"""What the calls of 8-bit buffers and of the gated block refuse, on the host, before anything is launched."""
import ctypes

import pytest

import paper_2603_05500_amd as px
from tests.test_abi import clib  # noqa: F401

FAR = [ctypes.c_void_p(0x10000000 * (i + 1)) for i in range(10)]      # never dereferenced; 256 MB apart


def at(p, bytes_on):
    return ctypes.c_void_p(p.value + bytes_on)


def test_mx8_refusals(clib):  # noqa: F811
    assert px.poetx_mx8_bytes(3, 130) == 768 + 3 * 8          # 3 rows of 256 codes, then two words of scales each
    assert px.poetx_mx8_bytes(0, 128) == px.poetx_mx8_bytes(1, 0) == px.poetx_mx8_bytes(-1, 5) == 0
    x, q = FAR[0], FAR[1]
    for f in (lambda **k: clib.poetx_mx8_quantize(k["x"], k["dt"], k["rows"], k["cols"], k["ld"], k["q"], None),
              lambda **k: clib.poetx_mx8_dequantize(k["q"], k["rows"], k["cols"], k["dt"], k["x"], k["ld"], None)):
        ok = dict(x=x, q=q, dt=px.BF16, rows=4, cols=64, ld=64)
        assert f(**{**ok, "x": None}) == 1 and f(**{**ok, "q": None}) == 1 and f(**{**ok, "dt": 2}) == 1
        assert f(**{**ok, "rows": 0}) == 1 and f(**{**ok, "cols": 0}) == 1 and f(**{**ok, "ld": 63}) == 2
        assert f(**{**ok, "q": at(q, 8)}) == 1                  # not 16-byte aligned
        assert f(**{**ok, "q": at(x, 64)}) == 1                 # overlaps
        assert f(**{**ok, "rows": 1 << 30, "ld": 1 << 20}) == 4


def _desc(**k):
    d = dict(d_in=256, d_hidden=512, groups=4, rows=100, dtype=px.BF16, activation=px.GATED_SILU, flags=0)
    d.update(k)
    return px.make_gated_desc(**d)


@pytest.mark.parametrize("bad,status", [(dict(d_in=0), 1), (dict(d_hidden=-1), 1), (dict(groups=0), 1), (dict(rows=-1), 1), (dict(dtype=7), 1), (dict(flags=4), 1),
                                        (dict(activation=2), 1), (dict(activation=-1), 1), (dict(flags=px.GATED_W_MX4, dtype=px.F32), 4), (dict(rows=1 << 30), 4),
                                        (dict(d_in=1 << 24), 4), (dict(d_hidden=1 << 23), 4), (dict(groups=1 << 22, d_hidden=1 << 9), 4)])
def test_gated_descriptors(clib, bad, status):  # noqa: F811
    d = _desc(**bad)
    assert px.poetx_gated_workspace_bytes(d) == 0
    p, big, ld = ctypes.byref(d), 1 << 62, 1 << 25
    f = FAR
    assert clib.poetx_gated_fwd(p, f[0], ld, f[1], f[2], f[3], ld, f[4], f[5], ld, f[6], big, None) == status
    assert clib.poetx_gated_bwd(p, f[0], ld, f[1], f[2], ld, f[3], f[4], f[5], ld, f[6], ld, None) == status
    assert clib.poetx_gated_bwd_recompute(p, f[0], ld, f[1], ld, f[2], f[3], f[4], f[5], ld, f[6], ld, f[7], big, None) == status


def test_gated_forward_arguments(clib):  # noqa: F811
    X, W, off, H, G, U, ws = FAR[:7]

    def fwd(d=None, flags=0, X=X, ldx=256, W=W, off=off, H=H, ldh=512, G=G, U=U, ldgu=512, ws=ws, n=1 << 40):
        return clib.poetx_gated_fwd(ctypes.byref(d or _desc(flags=flags)), X, ldx, W, off, H, ldh, G, U, ldgu, ws, n, None)

    assert fwd(X=None) == fwd(W=None) == fwd(off=None) == fwd(H=None) == 1
    assert fwd(G=None) == fwd(U=None) == 1                                    # one of a pair
    assert fwd(ldx=255) == fwd(ldh=511) == fwd(ldgu=511) == 2
    assert fwd(ldx=1 << 40) == fwd(ldh=1 << 40) == fwd(ldgu=1 << 40) == 4
    assert fwd(H=X) == fwd(H=W) == fwd(H=off) == fwd(G=X) == fwd(U=W) == fwd(G=H) == fwd(U=H) == fwd(U=G) == 1
    assert fwd(H=at(X, 2 * (99 * 256 + 255))) == 1                            # X's last element
    assert fwd(U=at(G, 2 * 511), ldgu=1024) == fwd(U=at(G, 2 * (1024 + 513)), ldgu=1024) == 1      # shares an element of each row
    four, both = px.GATED_W_MX4, px.GATED_W_MX4 | px.GATED_HELD_MX8
    assert fwd(flags=four, W=at(W, 8)) == 1
    assert fwd(flags=both, G=at(G, 8)) == fwd(flags=both, U=at(U, 4)) == fwd(flags=both, U=at(G, 512 * 100)) == 1
    many = _desc(flags=four, rows=4096)      # more rows than the kernels for a handful take
    need = px.poetx_gated_workspace_bytes(many)
    assert need > 0 and fwd(d=many, ws=None) == fwd(d=many, n=need - 1) == fwd(d=many, ws=at(ws, 8)) == 5
    assert fwd(d=many, ws=X) == fwd(d=many, ws=H) == fwd(d=many, ws=at(G, 16)) == 1
    # no rows: nothing to do, nothing looked at
    assert fwd(d=_desc(rows=0), X=None, H=None, G=None, U=None, ws=None, n=0) == 0


def test_gated_backward_arguments(clib):  # noqa: F811
    dH, G, U, off, dG, dU, H, X, W, ws = FAR

    def bwd(flags=0, rows=100, dH=dH, lddh=512, G=G, U=U, ldgu=512, off=off, dG=dG, dU=dU, lddgu=512, H=H, ldh=512):
        return clib.poetx_gated_bwd(ctypes.byref(_desc(flags=flags, rows=rows)), dH, lddh, G, U, ldgu, off, dG, dU, lddgu, H, ldh, None)

    def again(flags=0, rows=100, dH=dH, lddh=512, X=X, ldx=256, W=W, off=off, dG=dG, dU=dU, lddgu=512, H=H, ldh=512, ws=ws, n=1 << 40):
        return clib.poetx_gated_bwd_recompute(ctypes.byref(_desc(flags=flags, rows=rows)), dH, lddh, X, ldx, W, off, dG, dU, lddgu, H, ldh, ws, n, None)

    for f in (bwd, again):
        assert f(dH=None) == f(off=None) == f(dG=None) == f(dU=None) == 1
        assert f(lddh=511) == f(lddgu=511) == f(ldh=511) == 2
        assert f(lddh=1 << 40) == f(lddgu=1 << 40) == f(ldh=1 << 40) == 4
        assert f(dG=dH) == f(dU=dH) == f(H=dH) == f(H=off) == f(H=dG) == f(dU=H) == f(dU=dG) == 1
        assert f(dU=at(dG, 2 * 511), lddgu=1024) == 1
    assert bwd(G=None) == bwd(U=None) == 1 and bwd(ldgu=511) == 2
    assert bwd(dG=G) == bwd(dU=U) == bwd(H=G) == 1                            # in place
    assert bwd(flags=px.GATED_HELD_MX8, G=at(G, 8)) == bwd(flags=px.GATED_HELD_MX8, U=at(U, 8)) == 1
    assert again(X=None) == again(W=None) == 1 and again(ldx=255) == 2
    assert again(dG=X) == again(H=W) == 1
    four = px.GATED_W_MX4
    need = px.poetx_gated_workspace_bytes(_desc(flags=four, rows=4096))
    assert again(flags=four, rows=4096, ws=None) == again(flags=four, rows=4096, n=need - 1) == 5
    assert again(flags=four, rows=4096, ws=dH) == again(flags=four, rows=4096, ws=dU) == 1
    assert bwd(rows=0, dH=None, G=None, U=None, dG=None, dU=None, H=None) == 0
    assert again(rows=0, dH=None, X=None, dG=None, dU=None, H=None, ws=None, n=0) == 0


def test_weight_gradient_of_mx8_rows(clib):  # noqa: F811
    X, dZ, off, dW, ws = FAR[:5]
    g = lambda **k: px.make_grouped_desc(**{**dict(d_in=256, d_out=512, groups=4, rows=100, dtype=px.BF16, flags=px.GROUPED_X_MX8), **k})      # noqa: E731

    def f(d=None, X=X, ldx=0, lddz=512, dW=dW, ws=ws, n=1 << 40):
        return clib.poetx_grouped_bwd_weight(ctypes.byref(d or g()), X, ldx, dZ, lddz, off, dW, 0, ws, n, None)

    need = px.poetx_grouped_workspace_bytes(g())
    assert need >= 100 * 256 * 2
    assert f(ws=None) == f(n=need - 1) == f(ws=at(ws, 8)) == 5
    assert f(X=at(X, 8)) == f(ws=X) == f(ws=dZ) == f(ws=dW) == f(dW=X) == f(dW=dZ) == 1 and f(lddz=511) == 2
    assert f(d=g(flags=px.GROUPED_X_MX8 | px.GROUPED_W_MX4)) == 4             # a frozen weight has no gradient
    assert f(d=g(flags=px.GROUPED_X_MX8 | px.GROUPED_X_MX4 | px.GROUPED_W_MX4)) == 1
    p = ctypes.byref(g())
    assert clib.poetx_grouped_fwd(p, X, 256, dZ, off, dW, 512, ws, 1 << 40, None) == 4
    assert clib.poetx_grouped_bwd_input(p, X, 512, dZ, off, dW, 256, ws, 1 << 40, None) == 4
