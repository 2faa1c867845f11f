"""What the calls of 4-bit buffers, grouped products and group orders refuse, on the host, before anything is launched."""
import ctypes

import pytest

import paper_2603_05500_amd as px
from tests.test_abi import clib  # noqa: F401

FAR = [ctypes.c_void_p(0x10000000 * (i + 1)) for i in range(6)]      # never dereferenced; 256 MB apart


def test_mx4_refusals(clib):  # noqa: F811
    assert px.poetx_mx4_bytes(3, 130) == 512 + 3 * 8          # 3 rows of 256 codes: 384 bytes, then two words of scales each
    assert px.poetx_mx4_bytes(0, 128) == px.poetx_mx4_bytes(1, 0) == px.poetx_mx4_bytes(-1, 5) == 0
    x, q = FAR[0], FAR[1]
    for f in (lambda **k: clib.poetx_mx4_quantize(k["x"], k["dt"], k["rows"], k["cols"], k["ld"], k["q"], None),
              lambda **k: clib.poetx_mx4_dequantize(k["q"], k["rows"], k["cols"], k["dt"], k["x"], k["ld"], None)):
        ok = dict(x=x, q=q, dt=px.BF16, rows=4, cols=64, ld=64)
        assert f(**{**ok, "x": None}) == 1 and f(**{**ok, "q": None}) == 1 and f(**{**ok, "dt": 2}) == 1
        assert f(**{**ok, "rows": 0}) == 1 and f(**{**ok, "cols": 0}) == 1 and f(**{**ok, "ld": 63}) == 2
        assert f(**{**ok, "q": ctypes.c_void_p(FAR[1].value + 8)}) == 1                  # not 16-byte aligned
        assert f(**{**ok, "q": ctypes.c_void_p(FAR[0].value + 64)}) == 1                 # overlaps
        assert f(**{**ok, "rows": 1 << 30, "ld": 1 << 20}) == 4


def _desc(**k):
    d = dict(d_in=256, d_out=512, groups=4, rows=100, dtype=px.BF16, flags=0)
    d.update(k)
    return px.make_grouped_desc(**d)


@pytest.mark.parametrize("bad,status", [(dict(d_in=0), 1), (dict(d_out=-1), 1), (dict(groups=0), 1), (dict(rows=-1), 1), (dict(dtype=7), 1), (dict(flags=8), 1),
                                        (dict(flags=px.GROUPED_X_MX4), 1), (dict(flags=px.GROUPED_W_MX4, dtype=px.F32), 4), (dict(rows=1 << 30), 4),
                                        (dict(d_in=1 << 24), 4), (dict(groups=1 << 22, d_out=1 << 10), 4)])
def test_grouped_descriptors(clib, bad, status):  # noqa: F811
    d = _desc(**bad)
    assert px.poetx_grouped_workspace_bytes(d) == 0
    p = ctypes.byref(d)
    big = 1 << 62
    assert clib.poetx_grouped_fwd(p, FAR[0], 1 << 25, FAR[1], FAR[2], FAR[3], 1 << 25, FAR[4], big, None) == status
    assert clib.poetx_grouped_bwd_input(p, FAR[0], 1 << 25, FAR[1], FAR[2], FAR[3], 1 << 25, FAR[4], big, None) == status
    assert clib.poetx_grouped_bwd_weight(p, FAR[0], 1 << 25, FAR[1], 1 << 25, FAR[2], FAR[3], 0, FAR[4], big, None) == status


def test_grouped_arguments(clib):  # noqa: F811
    p = ctypes.byref(_desc())
    X, W, off, Z, ws = FAR[:5]

    def fwd(desc=p, X=X, ldx=256, W=W, off=off, Z=Z, ldz=512, ws=ws, n=1 << 40):
        return clib.poetx_grouped_fwd(desc, X, ldx, W, off, Z, ldz, ws, n, None)

    assert fwd(desc=None) == fwd(X=None) == fwd(W=None) == fwd(off=None) == fwd(Z=None) == 1
    assert fwd(ldx=255) == fwd(ldz=511) == 2
    assert fwd(Z=X) == fwd(Z=W) == fwd(Z=off) == 1
    assert fwd(Z=ctypes.c_void_p(X.value + 2 * (99 * 256 + 255))) == 1        # X's last element
    reserved = _desc()
    reserved.reserved = 1
    assert fwd(desc=ctypes.byref(reserved)) == 1
    q = ctypes.byref(_desc(flags=px.GROUPED_W_MX4 | px.GROUPED_X_MX4))
    need = px.poetx_grouped_workspace_bytes(_desc(flags=px.GROUPED_W_MX4 | px.GROUPED_X_MX4))
    assert need > 0 and fwd(desc=q, ws=None) == fwd(desc=q, n=need - 1) == 5
    assert clib.poetx_grouped_bwd_weight(q, X, 256, W, 512, off, Z, 0, ws, 1 << 40, None) == 4      # a frozen weight has no gradient
    assert clib.poetx_grouped_bwd_weight(p, X, 256, W, 511, off, Z, 0, ws, 1 << 40, None) == 2
    assert clib.poetx_grouped_bwd_weight(p, X, 256, W, 512, off, X, 0, ws, 1 << 40, None) == 1
    assert clib.poetx_grouped_bwd_weight(p, X, 256, W, 512, off, None, 0, ws, 1 << 40, None) == 1
    # no rows: nothing to do, nothing looked at
    none = ctypes.byref(_desc(rows=0))
    assert clib.poetx_grouped_fwd(none, None, 256, W, off, None, 512, None, 0, None) == 0
    assert clib.poetx_grouped_bwd_input(none, None, 512, W, off, None, 256, None, 0, None) == 0


def test_group_order_arguments(clib):  # noqa: F811
    ids, off, order, ws = FAR[:4]
    f = clib.poetx_group_order
    assert f(None, 5, 3, off, order, ws, 1 << 20, None) == f(ids, 5, 3, None, order, ws, 1 << 20, None) == f(ids, 5, 3, off, None, ws, 1 << 20, None) == 1
    assert f(ids, -1, 3, off, order, ws, 1 << 20, None) == f(ids, 5, 0, off, order, ws, 1 << 20, None) == 1
    assert f(ids, 5, 513, off, order, ws, 1 << 20, None) == 4
    assert f(ids, 5, 3, off, ids, ws, 1 << 20, None) == f(ids, 5, 3, ids, order, ws, 1 << 20, None) == 1
    need = px.poetx_group_order_workspace_bytes(1 << 20, 64)
    assert need > 0 and f(ids, 1 << 20, 64, off, order, None, 0, None) == f(ids, 1 << 20, 64, off, order, ws, need - 1, None) == 5
    assert px.poetx_group_order_workspace_bytes(8, 64) == 0 and px.poetx_group_order_workspace_bytes(8, 513) == 0
