"""Strides that a call of the gated block has no use for choose no kernel."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_gated import Block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,m,n,dtype,weight", [([2000, 0, 3561], 736, 328, "bf16", "dense"), ([1590, 1593], 4352, 40, "bf16", "dense"), ([3000, 1940], 512, 448, "f32", "dense"),
                                                     ([1031, 2000, 2000], 488, 336, "bf16", "mx4")])
def test_strides_that_are_not_used(lib, counts, m, n, dtype, weight):
    """ldgu of 8-bit buffers or of nothing, and ldh of no H, change nothing."""
    b = Block(counts, m, n, dtype, weight=weight)
    clib = px.load_library()
    pointer = lambda t: None if t is None else t.data_ptr()      # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    for flags, G, U in ((0, None, None), (px.GATED_HELD_MX8, *(torch.zeros(px.poetx_mx8_bytes(b.rows, b.n), dtype=torch.uint8, device="cuda") for _ in range(2)))):
        desc, results = b.desc(flags), []
        for unused in (0, -5, 1 << 30):
            ws, H = b.ws(desc), torch.zeros((b.rows, b.n), dtype=b.dt, device="cuda")
            dG, dU = torch.zeros((b.rows, 2 * b.n), dtype=b.dt, device="cuda").split(b.n, 1)
            size = 0 if ws is None else ws.numel()
            assert clib.poetx_gated_fwd(ctypes.byref(desc), b.X.data_ptr(), b.X.stride(0), b.W.data_ptr(), b.off.data_ptr(), H.data_ptr(), b.n, pointer(G), pointer(U), unused, pointer(ws), size, stream) == 0
            assert clib.poetx_gated_bwd_recompute(ctypes.byref(desc), b.dH.data_ptr(), b.dH.stride(0), b.X.data_ptr(), b.X.stride(0), b.W.data_ptr(), b.off.data_ptr(), dG.data_ptr(), dU.data_ptr(), 2 * b.n,
                                                  None, unused, pointer(ws), size, stream) == 0
            results.append([H, dG, dU] + ([] if G is None else [G.clone(), U.clone()]))
        for other in results[1:]:
            assert all(torch.equal(x, y) for x, y in zip(results[0], other)), flags
