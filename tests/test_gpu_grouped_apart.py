"""What one group holds stays out of the others' results, and a call repeated gives the same bits, on every kernel of the grouped calls."""
from __future__ import annotations

import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_grouped import CODE, DT, offsets_of, quantised, spread

pytestmark = pytest.mark.gpu

CALLS = [
    # dtype, weight, act, counts, d_in, d_out
    ("bf16", "dense", "same", [9, 0, 30, 21], 128, 136), ("f32", "dense", "same", [9, 0, 30, 21], 128, 136),                                     # a handful of rows
    ("bf16", "dense", "same", [300, 0, 77, 640], 130, 514), ("f32", "dense", "same", [300, 0, 77, 640], 130, 514),                               # edges
    ("bf16", "dense", "same", spread(8, 5000), 1032, 3000), ("bf16", "dense", "same", spread(64, 6000), 520, 1376), ("f32", "dense", "same", spread(8, 3000), 512, 768),
    ("bf16", "dense", "same", [200, 0, 300, 37, 251], 7808, 1248), ("bf16", "dense", "same", [500, 607], 776, 6368),                             # split contractions
    ("f32", "dense", "same", [500, 0, 640], 1760, 576), ("f32", "dense", "same", [100, 0, 140], 516, 2692),
    ("bf16", "mx4", "same", spread(64, 300), 256, 1376), ("bf16", "mx4", "same", spread(16, 8192), 512, 512), ("bf16", "mx4", "same", spread(8, 106), 11848, 640),
    ("bf16", "mx4", "same", [300, 0, 77, 640], 200, 1508),
    ("bf16", "mx4", "mx4", spread(64, 300), 256, 1376), ("bf16", "mx4", "mx4", spread(8, 5000), 1032, 3000), ("bf16", "mx4", "mx4", [300, 0, 77, 640], 200, 1508),
]


@pytest.mark.parametrize("dtype,weight,act,counts,m,n", CALLS)
def test_groups_are_apart(lib, dtype, weight, act, counts, m, n):
    G, rows, dt = len(counts), sum(counts), DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(m + n)
    off = offsets_of(counts)
    X, dZ = (torch.randn((rows, d), device="cuda", generator=g).to(dt) for d in (m, n))
    W = (torch.randn((G, n, m), device="cuda", generator=g) * 0.02).to(dt)
    desc = px.make_grouped_desc(m, n, G, rows, CODE[dtype], (px.GROUPED_W_MX4 if weight == "mx4" else 0) | (px.GROUPED_X_MX4 if act == "mx4" else 0))

    def results(fill):
        ws = torch.full((max(256, px.poetx_grouped_workspace_bytes(desc)),), fill, dtype=torch.uint8, device="cuda")
        Wx = quantised(W.view(G * n, m)) if weight == "mx4" else W
        Z, dX = torch.zeros((rows, n), dtype=dt, device="cuda"), torch.zeros((rows, m), dtype=dt, device="cuda")
        px.poetx_grouped_fwd(desc, X, Wx, off, Z, ws)
        px.poetx_grouped_bwd_input(desc, dZ, Wx, off, dX, ws)
        dW = None
        if weight == "dense":
            dW = torch.empty((G, n, m), device="cuda")
            px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False, ws)
        return Z, dX, dW

    once = results(0)
    again = results(255)
    assert all(torch.equal(a, b) for a, b in zip(once, again) if a is not None)
    k = max(range(G), key=lambda i: counts[i])                      # everything of the largest group becomes something else, then not finite
    a, b = int(off[k]), int(off[k + 1])
    for other in ("finite", "nan"):
        for t in (X[a:b], dZ[a:b], W[k]):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g) if other == "finite" else torch.full_like(t, float("nan")))
        then = results(0)
        for was, now in zip(once[:2], then[:2]):
            assert torch.equal(was[:a], now[:a]) and torch.equal(was[b:], now[b:]), other
            assert not torch.equal(was[a:b], now[a:b])
        if weight == "dense":
            assert torch.equal(once[2][:k], then[2][:k]) and torch.equal(once[2][k + 1:], then[2][k + 1:]), other


@pytest.mark.parametrize("counts,m,n", [([9, 0, 30, 21], 392, 136), ([300, 0, 77, 640], 392, 1512), ([300, 0, 77, 640], 392, 1508)])      # few rows; streamed codes; values
def test_both_in_four_bits_not_finite(lib, counts, m, n):
    """An infinity or NaN makes its block of 32 NaN: all of its row of Z, and the weight's its column of the group's rows."""
    G, rows = len(counts), sum(counts)
    off = offsets_of(counts)
    ends = off.tolist()
    g = torch.Generator(device="cuda").manual_seed(7)
    X = torch.randn((rows, m), device="cuda", generator=g).bfloat16()
    W = (torch.randn((G, n, m), device="cuda", generator=g) * 0.02).bfloat16()
    bad_rows = (ends[1] - 1, ends[2], ends[4] - 1)
    X[bad_rows[0], m - 1], X[bad_rows[1], 0], X[bad_rows[2], 128] = float("nan"), float("inf"), float("-inf")
    W[1] = float("nan")                                             # of a group without rows
    W[2, n - 1, m - 1], W[0, 0, 5] = float("nan"), float("inf")
    desc = px.make_grouped_desc(m, n, G, rows, px.BF16, px.GROUPED_W_MX4 | px.GROUPED_X_MX4)
    ws = torch.full((px.poetx_grouped_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    Z = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    px.poetx_grouped_fwd(desc, X, quantised(W.view(G * n, m)), off, Z, ws)
    want = torch.zeros_like(Z, dtype=torch.bool)
    for r in bad_rows:
        want[r] = True
    want[ends[2]: ends[3], n - 1] = want[: ends[1], 0] = True
    assert torch.equal(torch.isnan(Z), want) and bool(torch.isfinite(Z[~want]).all())
