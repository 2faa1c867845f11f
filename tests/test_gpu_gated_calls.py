"""How the block is called, on every one of its kernels: repeated, on another stream, captured; two captured passes with one workspace; NaN and infinities; rows beyond 2^31 elements."""
from __future__ import annotations

import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_gated import Block, _calls, scratch
from tests.test_gpu_gated_offsets import KERNELS

pytestmark = pytest.mark.gpu


def counts_of(groups, rows):
    """Uneven, and the second of more than two groups has no rows."""
    share = [0 if g == 1 and groups > 2 else 2 + g % 3 for g in range(groups)]
    counts = [rows * s // sum(share) for s in share]
    counts[-1] += rows - sum(counts)
    return counts


def block_of(kernel, seed=0):
    groups, rows, m, n, dtype, weight = KERNELS[kernel]
    return Block(counts_of(groups, rows), m, n, dtype, "silu" if n % 2 else "gelu", weight, seed=seed)


@pytest.mark.parametrize("kernel", KERNELS)
def test_repeated_on_another_stream_and_in_a_graph(lib, kernel):
    """The same bits every time."""
    run, outs = _calls(block_of(kernel))
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]

    def cleared():
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()

    def same(what):
        torch.cuda.synchronize()
        for i, (t, w) in enumerate(zip(outs, want)):
            assert torch.equal(t, w), (what, i)

    cleared()
    run()
    same("again")
    cleared()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    same("side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        cleared()
        graph.replay()
        same(f"replay {i}")
        run()      # eager work between replays
        same(f"eager {i}")


@pytest.mark.parametrize("kernel", ["in ranges", "in ranges narrow", "laid anew 256 x 128", "laid anew 256 narrow", "in ranges f32", "laid anew f32", "laid anew in ranges f32",
                                    "decoded in ranges", "decoded laid anew", "decoded laid anew in ranges", "few mx4 laid anew", "written out", "written out narrow"])
def test_two_graphs_share_a_workspace(lib, kernel):
    """Two captured passes over different rows and weights, forward and backward, with one workspace, replayed in turn on one stream."""
    blocks = [block_of(kernel, seed) for seed in (0, 1)]
    desc, mx8 = blocks[0].desc(), blocks[0].desc(px.GATED_HELD_MX8)
    assert px.poetx_gated_workspace_bytes(desc) == px.poetx_gated_workspace_bytes(mx8) > 0
    ws = scratch(px.poetx_gated_workspace_bytes(desc))
    outs, graphs, want = [], [], []
    for b in blocks:
        H, A = (torch.zeros((b.rows, b.n), dtype=b.dt, device="cuda") for _ in range(2))
        GU = torch.zeros((b.rows, 2 * b.n), dtype=b.dt, device="cuda")
        Q = [torch.zeros(px.poetx_mx8_bytes(b.rows, b.n), dtype=torch.uint8, device="cuda") for _ in range(2)]

        def run():
            px.poetx_gated_fwd(mx8, b.X, b.W, b.off, H, *Q, ws=ws)
            px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, *GU.split(b.n, 1), A, ws=ws)

        run()
        want.append([t.clone() for t in (H, A, GU, *Q)])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        outs.append((H, A, GU, *Q))
        graphs.append(g)
    assert not torch.equal(want[0][0], want[1][0])
    for _ in range(3):
        for t in (*outs[0], *outs[1]):
            t.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(t, w) for t, w in zip(outs[i], want[i])), i


@pytest.mark.parametrize("kernel", KERNELS)
def test_not_finite(lib, kernel):
    """NaN or an infinity of a row or of a group's weight stays in the elements that read it: the last column of gate and the first of up, whose rows are neighbours in memory, one row of X, and the
    whole weight of a group without rows."""
    b = block_of(kernel)
    m, n, groups = b.m, b.n, b.groups
    ends = b.off.tolist()
    rows = slice(ends[-2], ends[-1])                 # of the last group
    nan = float("nan")
    if b.flags:                                      # scale 255: 32 values that are NaN
        pitch = -(-m // 128) * 4
        scales = b.W[-(-groups * 2 * n * pitch * 16 // 256) * 256:][: groups * 2 * n * pitch].view(groups, 2 * n, pitch)
        scales[-1, n - 1, 0] = scales[-1, n, (m - 1) // 32] = 255
        if groups > 2:
            scales[1, :, : -(-m // 32)] = 255
    else:
        b.W[-1, n - 1, 0] = nan
        b.W[-1, n, m - 1] = float("inf")
        if groups > 2:
            b.W[1] = nan
    b.X[ends[1] - 1, m - 1] = nan
    of_G, of_U = (torch.zeros((b.rows, n), dtype=torch.bool, device="cuda") for _ in range(2))
    of_G[rows, n - 1] = of_U[rows, 0] = True
    of_G[ends[1] - 1] = of_U[ends[1] - 1] = True
    b.dH[ends[1] // 2, 3] = float("inf")
    of_dH = torch.zeros_like(of_G)
    of_dH[ends[1] // 2, 3] = True
    desc, mx8 = b.desc(), b.desc(px.GATED_HELD_MX8)
    H, G, U, dG, dU = (torch.zeros((b.rows, n), dtype=b.dt, device="cuda") for _ in range(5))
    bad = lambda t: ~torch.isfinite(t)      # noqa: E731
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, ws=b.ws(desc))
    assert torch.equal(bad(H), of_G | of_U)
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, G, U, ws=b.ws(desc))
    assert torch.equal(bad(H), of_G | of_U) and torch.equal(bad(G), of_G) and torch.equal(bad(U), of_U)
    px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, dG, dU, H, ws=b.ws(desc))
    assert torch.equal(bad(H), of_G | of_U) and torch.equal(bad(dG), of_G | of_U | of_dH) and torch.equal(bad(dU), of_G | of_dH)
    QG, QU = (torch.zeros(px.poetx_mx8_bytes(b.rows, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    px.poetx_gated_fwd(mx8, b.X, b.W, b.off, H, QG, QU, ws=b.ws(mx8))
    assert torch.equal(bad(H), of_G | of_U)
    for Q, of, t in ((QG, of_G, G), (QU, of_U, U)):
        px.poetx_mx8_dequantize(Q, t)
        blocks = torch.nn.functional.pad(of, (0, -n % 32)).view(b.rows, -1, 32).any(2)      # a block shares its NaN
        assert torch.equal(bad(t), blocks.repeat_interleave(32, 1)[:, :n])


@pytest.mark.parametrize("kernel", [k for k, s in KERNELS.items() if s[1] >= 1100])
def test_rows_past_32_bits(lib, kernel):
    """Matrices whose last rows begin beyond 2^31 elements: the same bits as close together, and nothing between the rows written."""
    b = block_of(kernel)
    rows, m, n, dt = b.rows, b.m, b.n, b.dt
    odd = n % 8 != 0
    ld = -(-2 ** 31 // (rows - 40) // 64) * 64 + (1 if odd else 0)
    assert (rows - 40) * ld >= 2 ** 31 - ld
    step = n if odd else -(-n // 8) * 8
    flat, pairs = (torch.full((rows, ld), 3.0, dtype=dt, device="cuda") for _ in range(2))      # no output of a call lies between the rows of another but its own pair's
    (H, A), (G, U, dG, dU) = ([t[:, 64 + step * i: 64 + step * i + n] for i in range(k)] for t, k in ((flat, 2), (pairs, 4)))
    Xw = torch.zeros((rows, -(-ld // 64) * 64), dtype=dt, device="cuda")
    X, dH = Xw[:, :m], Xw[:, -(-m // 64) * 64:][:, :n]
    X.copy_(b.X)
    dH.copy_(b.dH)
    desc = b.desc()
    close = [torch.zeros((rows, n), dtype=dt, device="cuda") for _ in range(6)]
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, close[0], close[1], close[2], ws=b.ws(desc))
    px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, close[3], close[4], close[5], ws=b.ws(desc))
    px.poetx_gated_fwd(desc, X, b.W, b.off, H, G, U, ws=b.ws(desc))
    px.poetx_gated_bwd_recompute(desc, dH, X, b.W, b.off, dG, dU, A, ws=b.ws(desc))
    for name, got, want in zip(("H", "G", "U", "dG", "dU", "H again"), (H, G, U, dG, dU, A), close):
        assert torch.equal(got, want), name
        got.fill_(3.0)
    assert all(bool((part == 3.0).all()) for t in (flat, pairs) for part in t.split(256)), "written between the rows"
