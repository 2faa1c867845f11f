"""Offsets that are not in order, or point outside the rows: every kernel of the grouped calls gives every row the group that the header says, and touches nothing else.

The oracle takes offsets inside 0 .. rows and none below those before it, so that group g has the rows from the largest of offsets[0 .. g] to the largest of offsets[0 .. g + 1]; for
the weight gradient from offsets[g] to offsets[g + 1].
Bounds as in test_gpu_grouped.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_grouped import CODE, DT, quantised, reference, strided, within

pytestmark = pytest.mark.gpu


def disorder(kind, groups, rows):
    """groups + 1 int32 offsets."""
    rng = np.random.default_rng(groups + rows)
    off = np.sort(rng.integers(0, rows + 1, groups + 1))
    if kind == "back and forth":              # most rows claimed by several pairs, the last tenth by one
        off = np.where(np.arange(groups + 1) % 2, rows * 9 // 10, 0)
        off[-1] = rows
    elif kind == "some anywhere":
        off[1::3] = rng.integers(0, rows + 1, len(off[1::3]))
    elif kind == "outside":
        off = off * 2 - rows // 2
        off[0], off[groups // 2], off[-1] = -2 ** 31, -7, 2 ** 31 - 1
    elif kind == "first in the middle":       # rows below it have pairs that name them, and no group
        off[0] = rows // 2
    elif kind == "last first":
        off = off[::-1].copy()
    elif kind == "below":
        off = off - rows - 1
    elif kind == "above":
        off = off + rows
    return off


KINDS = ["back and forth", "some anywhere", "outside", "first in the middle", "last first", "below", "above"]
CALLS = [
    # dtype, weight, act, groups, rows, d_in, d_out
    ("bf16", "dense", "same", 4, 100, 128, 128), ("f32", "dense", "same", 4, 100, 128, 128),                                              # a handful of rows
    ("bf16", "dense", "same", 5, 1000, 130, 258), ("f32", "dense", "same", 5, 1000, 130, 258),                                            # edges
    ("bf16", "dense", "same", 300, 2000, 128, 136),
    ("bf16", "dense", "same", 8, 5000, 1032, 3000), ("bf16", "dense", "same", 64, 6000, 520, 1376), ("bf16", "dense", "same", 200, 3000, 256, 512),      # streams
    ("f32", "dense", "same", 8, 3000, 512, 768), ("bf16", "dense", "same", 5, 788, 7808, 1248), ("f32", "dense", "same", 3, 1140, 1760, 576),            # split contractions
    ("bf16", "mx4", "same", 64, 300, 256, 1376), ("bf16", "mx4", "same", 5, 700, 1032, 1000), ("bf16", "mx4", "same", 16, 8192, 512, 512),               # 4-bit weights
    ("bf16", "mx4", "same", 4, 5000, 2600, 2072), ("bf16", "mx4", "same", 8, 106, 11848, 640), ("bf16", "mx4", "same", 4, 3000, 200, 500),
    ("bf16", "mx4", "mx4", 64, 300, 256, 1376), ("bf16", "mx4", "mx4", 8, 5000, 1032, 3000), ("bf16", "mx4", "mx4", 4, 3000, 200, 500),                  # both
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,weight,act,groups,rows,m,n", CALLS)
def test_offsets_not_in_order(lib, dtype, weight, act, groups, rows, m, n, kind):
    offsets = disorder(kind, groups, rows)
    ends = np.maximum.accumulate(np.clip(offsets, 0, rows))
    counts, first, last = np.diff(ends).tolist(), int(ends[0]), int(ends[-1])
    off, dt = torch.from_numpy(offsets.astype(np.int32)).cuda(), DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(groups + rows)
    X, dZ = (torch.full((rows, d), float("nan"), device="cuda", dtype=dt) for d in (m, n))      # rows of no group stay NaN
    for t in (X, dZ):
        t[first: last] = torch.randn((last - first, t.shape[1]), device="cuda", generator=g).to(dt)
    W = (torch.randn((groups, n, m), device="cuda", generator=g) * 0.02).to(dt)
    Wx, Xr, flags = W, X[first: last], 0
    if weight == "mx4":
        Wx, flags = quantised(W.view(groups * n, m)), px.GROUPED_W_MX4
        px.poetx_mx4_dequantize(Wx, W.view(groups * n, m))
    if act == "mx4":
        flags |= px.GROUPED_X_MX4
        if last > first:
            Xr = torch.empty_like(Xr)
            px.poetx_mx4_dequantize(quantised(X[first: last]), Xr)
    desc = px.make_grouped_desc(m, n, groups, rows, CODE[dtype], flags)
    ws = torch.full((max(256, px.poetx_grouped_workspace_bytes(desc)),), 255, dtype=torch.uint8, device="cuda")
    for call, x, xr, d, contraction, which in ((px.poetx_grouped_fwd, X, Xr, n, m, "fwd"), (px.poetx_grouped_bwd_input, dZ, dZ[first: last], m, n, "input")):
        out, flat = strided(rows, d, 8, dt, 8, fill=3.0)
        call(desc, x, Wx, off, out, ws)
        assert within(out[first: last], *reference(which, xr, W, counts), contraction, dtype), which
        out[first: last] = 3.0
        assert bool((flat == 3.0).all()), (which, "written where no group is")
    if weight == "dense":
        flat = torch.full((groups * n * m + 64,), 3.0, device="cuda")
        dW = flat[: groups * n * m].view(groups, n, m)
        for t in (X, dZ):
            t[torch.isnan(t)] = 0.5              # rows of no group may be named by a pair
        px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False, ws)
        for k in range(groups):                  # the rows that the group's own offsets name
            a, b = (int(e) for e in np.clip(offsets[k: k + 2], 0, rows))
            ref, mag = reference("weight", X[a:], None, [max(b - a, 0)], dZ[a:])
            assert within(dW[k], ref[0], mag[0], rows, "f32"), k
        assert bool((flat[groups * n * m:] == 3.0).all())


@pytest.mark.parametrize("groups,rows,m,n,before,behind", [(6, 200, 256, 384, 37, 90), (1, 9, 4096, 1024, 3, 5), (8, 4000, 1032, 3000, 100, 301),
                                                           (4, 3000, 200, 500, 1, 77)])      # few rows; streamed codes; values
def test_rows_of_no_group_leave_no_trace(lib, groups, rows, m, n, before, behind):
    """With both operands in four bits: what rows of no group hold shows neither in the output nor in the scratch."""
    total = before + rows + behind
    g = torch.Generator(device="cuda").manual_seed(rows)
    X = torch.randn((total, m), device="cuda", generator=g).bfloat16()
    Q = quantised((torch.randn((groups * n, m), device="cuda", generator=g) * 0.02).bfloat16())
    off = (torch.arange(groups + 1, device="cuda") * rows // groups + before).int()
    desc = px.make_grouped_desc(m, n, groups, total, px.BF16, px.GROUPED_W_MX4 | px.GROUPED_X_MX4)
    after = []
    for other in (0.0, 5.0):
        X[:before] = X[before + rows:] = other
        ws = torch.full((px.poetx_grouped_workspace_bytes(desc),), 170, dtype=torch.uint8, device="cuda")
        Z = torch.full((total, n), 3.0, dtype=torch.bfloat16, device="cuda")
        px.poetx_grouped_fwd(desc, X, Q, off, Z, ws)
        after.append((ws, Z))
    assert torch.equal(after[0][0], after[1][0]) and torch.equal(after[0][1], after[1][1])
    assert not bool((after[0][1][before: before + rows] == 3.0).all())
