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
