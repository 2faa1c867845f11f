"""What the calls of 8-bit rows refuse of their workspace, on the host."""
import ctypes

import paper_2603_05500_amd as px
from tests.test_abi import clib  # noqa: F401
from tests.test_gated_abi import FAR, at


def test_workspace_over_the_offsets(clib):  # noqa: F811
    """Values written into the workspace would change the offsets that the next kernels read."""
    X, dZ, off, dW, ws = FAR[:5]
    groups = 4
    d = px.make_grouped_desc(256, 512, groups, 100, px.BF16, px.GROUPED_X_MX8)
    need = px.poetx_grouped_workspace_bytes(d)
    assert need % 16 == 0
    for p in (off, at(off, 16 - need), at(off, 4 * (groups + 1) // 16 * 16)):      # the first, and each end's last 16 bytes that touch it
        assert clib.poetx_grouped_bwd_weight(ctypes.byref(d), X, 0, dZ, 512, off, dW, 0, p, 1 << 40, None) == 1
