"""Scratch and empty calls of the grouped products and the group order: what is refused on the host, and what is not."""
import ctypes

import paper_2603_05500_amd as px
from tests.test_abi import clib  # noqa: F401
from tests.test_grouped_abi import FAR


def at(p, off):
    return ctypes.c_void_p(p.value + off)


def test_group_order_scratch(clib):  # noqa: F811
    ids, off, order, ws = FAR[:4]
    n, groups = 1 << 20, 64
    need = px.poetx_group_order_workspace_bytes(n, groups)

    def call(ws):
        return clib.poetx_group_order(ids, n, groups, off, order, ws, need, None)

    assert call(at(ws, 2)) == 5                                                          # not a place for int32
    for p, nbytes in ((ids, 4 * n), (off, 4 * (groups + 1)), (order, 4 * n)):
        assert call(p) == call(at(p, nbytes - 4)) == call(at(p, 4 - need)) == 1


def test_no_rows(clib):  # noqa: F811
    """A call without rows looks at no row tensor, wherever its pointers point; the weight gradient still writes, and minds where."""
    X, W, off = FAR[:3]
    for flags in (0, px.GROUPED_W_MX4):
        p = ctypes.byref(px.make_grouped_desc(256, 512, 4, 0, px.BF16, flags))
        for out in (at(W, 64), at(off, 4), W, X):
            assert clib.poetx_grouped_fwd(p, X, 256, W, off, out, 512, None, 0, None) == 0
            assert clib.poetx_grouped_bwd_input(p, X, 512, W, off, out, 256, None, 0, None) == 0
    p = ctypes.byref(px.make_grouped_desc(256, 512, 4, 0, px.BF16, 0))
    assert clib.poetx_grouped_bwd_weight(p, None, 256, None, 512, off, at(off, 4), 0, None, 0, None) == 1
