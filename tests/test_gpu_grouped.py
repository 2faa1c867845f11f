"""4-bit buffers, grouped products and the order of groups against plain float64 forms written here.

Bounds.  A product of two bf16 (or of two 4-bit values) is exact in fp32, so a result differs from the exact sum by the
roundings of K fp32 additions, at most K 2^-24 of the sum of magnitudes (fp32 inputs: one rounding more per product), and by
one rounding to its own type: 2^-8 of itself in bf16 (8 significant bits, half a unit of the last), 2^-24 in fp32.  Conversions to and from four bits are exact."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2603_05500_amd as px

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": px.F32, "bf16": px.BF16}
GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def strided(rows, cols, pad, dtype, shift=0, fill=float("nan")):
    """A rows x cols matrix with `pad` columns between its rows and `shift` elements in front, all of them `fill`."""
    flat = torch.full((rows * (cols + pad) + shift + 8,), fill, dtype=dtype, device="cuda")
    return flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], flat


# ------------------------------------------------------------------------------------ four bits
def oracle_codes(x):
    """float64 [rows][cols] -> codes [rows][mp], scale bytes [rows][mp / 32], by the definition."""
    rows, cols = x.shape
    mp = -(-cols // 128) * 128
    code, scale = np.zeros((rows, mp), np.int64), np.zeros((rows, mp // 32), np.int64)
    p = np.zeros((rows, mp))
    p[:, :cols] = x
    for b in range(mp // 32):
        blk = p[:, 32 * b: 32 * b + 32]
        for r in range(rows):
            v = blk[r]
            if not np.isfinite(v).all():
                scale[r, b] = 255
                continue
            top = np.abs(v).max()
            if top == 0:
                code[r, 32 * b: 32 * b + 32] = 8 * np.signbit(v)
                continue
            s = min(max(int(np.floor(np.log2(top))) - 2 + 127, 0), 254)
            scale[r, b] = s
            a = np.abs(v) * 2.0 ** (127 - s)
            dist = np.abs(a[:, None] - GRID[None])
            c = dist.argmin(1)                      # the lower of two equally near ...
            tie = (c < 7) & (dist[np.arange(32), c] == dist[np.arange(32), np.minimum(c + 1, 7)])
            c = np.where(tie & (c % 2 == 1), c + 1, c)     # ... unless the upper one is even
            code[r, 32 * b: 32 * b + 32] = c + 8 * np.signbit(v)
    return code, scale


def oracle_values(code, scale, cols):
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale - 127.0))
    return (v * np.repeat(s, 32, axis=1))[:, :cols]


def split_buffer(Q, rows, cols):
    q = Q.cpu().numpy()
    mp = -(-cols // 128) * 128
    off = -(-rows * mp // 2 // 256) * 256
    b = q[: rows * mp // 2].reshape(rows, -1).astype(np.int64)
    code = np.stack([b & 15, b >> 4], -1).reshape(rows, mp)
    return code, q[off: off + rows * mp // 32].reshape(rows, -1).astype(np.int64)


def quantised(W, fill=255):
    """W (rows x cols on the device) -> its 4-bit buffer, which held `fill` before."""
    Q = torch.full((px.poetx_mx4_bytes(*W.shape),), fill, dtype=torch.uint8, device="cuda")
    px.poetx_mx4_quantize(W, Q)
    return Q


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 0), (2, 33, 7, 1), (4, 127, 1, 3), (7, 128, 8, 0), (17, 160, 0, 0),
                                                 (33, 257, 3, 1), (9, 1376, 0, 0), (1, 4096, 0, 0)])
def test_mx4_round_trip(lib, rows, cols, pad, shift, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-30, 30, (rows, 1)).astype(float))
    X, _ = strided(rows, cols, pad, DT[dtype], shift)
    X.copy_(dev(x, DT[dtype]))
    code, scale = oracle_codes(host(X))
    Q = quantised(X)
    got_c, got_s = split_buffer(Q, rows, cols)
    assert np.array_equal(got_s, scale) and np.array_equal(got_c, code)
    want = oracle_values(code, scale, cols)
    for out_type in ("bf16", "f32"):
        out, flat = strided(rows, cols, pad, DT[out_type], shift, fill=7.0)
        px.poetx_mx4_dequantize(Q, out)
        assert np.array_equal(host(out), want)
        left = flat.clone()
        left[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 7.0
        assert bool((left == 7.0).all()), "written outside the matrix"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mx4_ties_and_extremes(lib, dtype):
    """Every tie and its neighbours, zeros, the smallest and largest numbers, infinities and NaN."""
    tie = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7.5])
    rows = [np.concatenate([[4.0], tie[:7], -tie[:7], np.zeros(17)]), np.concatenate([[7.5, -7.5], tie, -tie, np.zeros(14)]),
            np.concatenate([[4.0], tie[:7] * (1 + 2.0 ** -7), tie[:7] * (1 - 2.0 ** -7), np.full(17, -0.0)]),
            np.zeros(32), np.full(32, -0.0), np.full(32, 2.0 ** -126), np.full(32, 2.0 ** -130), np.full(32, 3.0e38), np.arange(32) * 2.0 ** -133,
            np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.ones(7), np.nan, np.zeros(24)], np.r_[1e30, np.full(31, 1e-30)]]
    X = dev(np.array(rows), DT[dtype])
    code, scale = oracle_codes(host(X))
    Q = quantised(X)
    got_c, got_s = split_buffer(Q, *X.shape)
    assert np.array_equal(got_s, scale) and np.array_equal(got_c, code)
    out = torch.empty_like(X)
    px.poetx_mx4_dequantize(Q, out)
    assert np.array_equal(host(out), oracle_values(code, scale, 32), equal_nan=True)


def test_mx4_all_codes_and_scales(lib):
    """A buffer a caller built: every code under every scale byte, 2^-127 and NaN among them; what bf16 or fp32 cannot hold is infinite."""
    rows = 256
    code = np.tile(np.r_[np.arange(16), np.arange(16)[::-1]], (rows, 4))
    scale = np.tile(np.arange(256)[:, None], (1, 4))
    Q = torch.from_numpy(np.concatenate([(code[:, 0::2] + 16 * code[:, 1::2]).astype(np.uint8).ravel(), scale.astype(np.uint8).ravel()])).cuda()
    want = torch.from_numpy(oracle_values(code, scale, 128))
    for dtype in DT.values():
        out = torch.empty((rows, 128), dtype=dtype, device="cuda")
        px.poetx_mx4_dequantize(Q, out)
        assert np.array_equal(host(out), want.to(dtype).double().numpy(), equal_nan=True)


# ------------------------------------------------------------------------------------ grouped products
def offsets_of(counts):
    return torch.tensor(np.r_[0, np.cumsum(counts)], dtype=torch.int32, device="cuda")


def bound(mag, ref, K, dtype):
    return (K + 4) * 2.0 ** -24 * mag + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(ref) + 1e-37


def check(got, ref, mag, K, dtype, what):
    assert np.isfinite(got).all(), what
    err, lim = np.abs(got - ref), bound(mag, ref, K, dtype)
    assert (err <= lim).all(), (what, float(err.max()), float((err / lim).max()))


def run_grouped(counts, m, n, dtype, weight="dense", act="same", pads=(0, 0), shift=0, extra=0, kinds=("fwd", "input", "weight"), seed=0):
    """All the calls on groups of `counts` rows, with `extra` rows behind them that no group has, against float64."""
    rng = np.random.default_rng(seed + m + 7 * n + 31 * len(counts))
    G, rows, dt = len(counts), int(sum(counts)) + extra, DT[dtype]
    off = offsets_of(counts)
    ends = off.cpu().numpy()
    X, _ = strided(rows, m, pads[0], dt, shift)
    dZ, _ = strided(rows, n, pads[1], dt, shift)
    live = int(sum(counts))
    X[:live].copy_(dev(rng.standard_normal((live, m)), dt))       # the rows of no group stay NaN, as does what lies between rows
    dZ[:live].copy_(dev(rng.standard_normal((live, n)) * 0.1, dt))
    W = dev(rng.standard_normal((G, n, m)) * 0.02, dt)
    flags = 0
    Wx, Wh, Xh, dZh = W, host(W), host(X), host(dZ)
    if weight == "mx4":
        Wx, flags = quantised(W.view(G * n, m)), px.GROUPED_W_MX4
        Wh = oracle_values(*split_buffer(Wx, G * n, m), m).reshape(G, n, m)
    if act == "mx4":
        flags |= px.GROUPED_X_MX4
        q = quantised(X[:live].contiguous()) if live else None
        Xq = oracle_values(*split_buffer(q, live, m), m) if live else Xh
    desc = px.make_grouped_desc(m, n, G, rows, CODE[dtype], flags)
    need = px.poetx_grouped_workspace_bytes(desc)
    ws = torch.full((need // 4 + 64,), float("nan"), device="cuda").view(torch.uint8) if need else None
    res = {}
    if "fwd" in kinds:
        Z, flat = strided(rows, n, pads[1], dt, shift, fill=3.0)
        px.poetx_grouped_fwd(desc, X, Wx, off, Z, ws)
        ref, mag = np.full((rows, n), 3.0), np.zeros((rows, n))
        xs = Xq if act == "mx4" else Xh
        for g in range(G):
            a, b = ends[g], ends[g + 1]
            ref[a:b], mag[a:b] = xs[a:b] @ Wh[g].T, np.abs(xs[a:b]) @ np.abs(Wh[g]).T
        check(host(Z), ref, mag, m, dtype, "Z")
        Z.fill_(3.0)
        assert bool((flat == 3.0).all()), "Z: written outside the matrix"
        res["Z"] = Z
    if "input" in kinds:
        dX, flat = strided(rows, m, pads[0], dt, shift, fill=3.0)
        px.poetx_grouped_bwd_input(desc, dZ, Wx, off, dX, ws)
        ref, mag = np.full((rows, m), 3.0), np.zeros((rows, m))
        for g in range(G):
            a, b = ends[g], ends[g + 1]
            ref[a:b], mag[a:b] = dZh[a:b] @ Wh[g], np.abs(dZh[a:b]) @ np.abs(Wh[g])
        check(host(dX), ref, mag, n, dtype, "dX")
        dX.fill_(3.0)
        assert bool((flat == 3.0).all()), "dX: written outside the matrix"
    if "weight" in kinds and weight == "dense":
        dW = torch.full((G, n, m), float("nan"), device="cuda")
        px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False, ws)
        first = dW.clone()
        px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, True, ws)
        for g in range(G):
            a, b = ends[g], ends[g + 1]
            ref, mag = dZh[a:b].T @ Xh[a:b], np.abs(dZh[a:b]).T @ np.abs(Xh[a:b])
            check(host(first[g]), ref, mag, b - a, "f32", "dW")
            check(host(dW[g]), 2 * ref, 2 * mag, b - a, "f32", "dW added to")
    return res


SHAPES = [
    # counts, m, n
    ([1], 1, 1), ([0], 8, 8), ([3], 7, 5), ([1, 0, 2], 33, 17), ([5, 1, 0, 130, 64], 64, 96), ([31, 33, 32], 100, 60),
    ([0, 0, 7], 256, 128), ([257], 130, 258), ([128, 129, 127], 128, 256), ([300, 0, 1, 211], 256, 320), ([64] * 5, 96, 1376),
    ([1] * 70, 64, 64), ([2, 0] * 70, 40, 72), ([600, 5], 512, 264),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,m,n", SHAPES)
def test_grouped(lib, counts, m, n, dtype):
    run_grouped(counts, m, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pads,shift,extra", [((8, 16), 0, 0), ((3, 5), 0, 9), ((0, 0), 1, 0), ((8, 8), 8, 130), ((1, 0), 3, 1)])
def test_grouped_strides(lib, pads, shift, extra, dtype):
    run_grouped([17, 0, 150, 3], 136, 200, dtype, pads=pads, shift=shift, extra=extra)


@pytest.mark.parametrize("act", ["same", "mx4"])
@pytest.mark.parametrize("counts,m,n", SHAPES + [([1], 4096, 512), ([1, 1, 0, 1], 1024, 1376), ([16], 640, 256), ([17, 40], 2048, 264), ([513], 1408, 512)])
def test_grouped_mx4(lib, counts, m, n, act):
    run_grouped(counts, m, n, "bf16", weight="mx4", act=act)


@pytest.mark.parametrize("act", ["same", "mx4"])
@pytest.mark.parametrize("pads,shift,extra", [((8, 16), 0, 0), ((3, 5), 0, 9), ((0, 0), 1, 0), ((8, 8), 8, 130)])
def test_grouped_mx4_strides(lib, pads, shift, extra, act):
    run_grouped([17, 0, 150, 3], 136, 200, "bf16", weight="mx4", act=act, pads=pads, shift=shift, extra=extra)


@pytest.mark.parametrize("weight", ["dense", "mx4"])
def test_grouped_not_finite(lib, weight):
    """An infinity or NaN in one row or one group's weight stays in what reads it."""
    m, n, counts = 256, 256, [130, 70, 0, 300]
    G, rows = len(counts), sum(counts)
    off = offsets_of(counts)
    g = torch.Generator(device="cuda").manual_seed(3)
    X, dZ = (torch.randn((rows, d), device="cuda", generator=g).bfloat16() for d in (m, n))
    W = (torch.randn((G, n, m), device="cuda", generator=g) * 0.02).bfloat16()
    X[129, 255], X[200, 0], dZ[130, 3], dZ[199, 255] = float("nan"), float("inf"), float("nan"), float("-inf")
    W[2] = float("nan")                       # the weight of a group without rows
    W[3, 5, 7] = float("nan")
    Wx, flags = (quantised(W.view(G * n, m)), px.GROUPED_W_MX4) if weight == "mx4" else (W, 0)
    desc = px.make_grouped_desc(m, n, G, rows, px.BF16, flags)
    ws = torch.empty(max(256, px.poetx_grouped_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    Z, dX = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, m), dtype=torch.bfloat16, device="cuda")
    px.poetx_grouped_fwd(desc, X, Wx, off, Z, ws)
    px.poetx_grouped_bwd_input(desc, dZ, Wx, off, dX, ws)
    bad = ~torch.isfinite(Z)
    want = torch.zeros_like(bad)
    want[129] = want[200] = True
    want[200:, 5] = True
    assert torch.equal(bad, want)
    bad = ~torch.isfinite(dX)
    want = torch.zeros_like(bad)
    want[130] = want[199] = True
    cols = slice(0, 32) if weight == "mx4" else slice(7, 8)      # a block of four-bit values shares its NaN
    want[200:, cols] = True
    assert torch.equal(bad, want)
    if weight == "dense":
        dW = torch.empty((G, n, m), device="cuda")
        px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False, ws)
        bad = ~torch.isfinite(dW)
        want = torch.zeros_like(bad)
        want[0, :, 255] = want[1, 3] = want[1, 255] = want[3, :, 0] = True
        assert torch.equal(bad, want)


def test_grouped_offsets_out_of_range(lib):
    """Offsets past the rows, below zero or decreasing touch nothing outside the tensors; groups that are in order get their rows."""
    m = n = 128
    rows = 100
    X = torch.randn((rows, m), device="cuda").bfloat16()
    W = torch.randn((4, n, m), device="cuda").bfloat16()
    desc = px.make_grouped_desc(m, n, 4, rows, px.BF16)
    off = torch.tensor([-5, 40, 30, 70, 1000], dtype=torch.int32, device="cuda")
    flat = torch.full((rows + 64, n), 3.0, dtype=torch.bfloat16, device="cuda")
    Z = flat[:rows]
    px.poetx_grouped_fwd(desc, X, W, off, Z)
    ref = torch.empty((rows, n), dtype=torch.float64)
    for a, b, g in ((0, 30, 0), (40, 70, 2), (70, 100, 3)):      # rows 30 .. 39 are claimed twice
        ref[a:b] = X[a:b].double().cpu() @ W[g].double().cpu().t()
        assert float((Z[a:b].double().cpu() - ref[a:b]).abs().max()) <= 2.0 ** -8 * float(ref[a:b].abs().max())
    assert bool((flat[rows:] == 3.0).all())


def test_gradients_against_differences(lib):
    """dX and dW are the derivatives of L = <dZ, Z(X, W)>: Z is linear in either, so differences of any size are exact."""
    counts, m, n = [5, 0, 9], 24, 40
    G, rows = len(counts), sum(counts)
    off = offsets_of(counts)
    g = torch.Generator(device="cuda").manual_seed(1)
    X, dZ = (torch.randn((rows, d), device="cuda", generator=g) for d in (m, n))
    W = torch.randn((G, n, m), device="cuda", generator=g)
    desc = px.make_grouped_desc(m, n, G, rows, px.F32)
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    px.poetx_grouped_bwd_input(desc, dZ, W, off, dX)
    px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False)

    def loss(x, w):
        Z = torch.zeros((rows, n), device="cuda")
        px.poetx_grouped_fwd(desc, x, w, off, Z)
        return float((Z.double() * dZ.double()).sum())

    for i in range(6):
        vx, vw = torch.randn(X.shape, device="cuda", generator=g), torch.randn(W.shape, device="cuda", generator=g)
        size = float(vx.abs().sum() + vw.abs().sum())      # every product of the sums is of order one
        assert abs((loss(X + vx, W) - loss(X - vx, W)) / 2 - float((dX.double() * vx.double()).sum())) < 1e-6 * size * n
        assert abs((loss(X, W + vw) - loss(X, W - vw)) / 2 - float((dW.double() * vw.double()).sum())) < 1e-6 * size * n


def test_results_do_not_depend_on_the_other_groups(lib):
    """A group's rows and weight give the same bits again on a second call."""
    for dtype in ("bf16", "f32"):
        a = run_grouped([300, 0, 77, 140], 256, 512, dtype, kinds=("fwd",))["Z"]
        X = torch.randn((517, 256), device="cuda").to(DT[dtype])
        dZ = torch.randn((517, 512), device="cuda").to(DT[dtype])
        desc = px.make_grouped_desc(256, 512, 4, 517, CODE[dtype])
        off = offsets_of([300, 0, 77, 140])
        dW = [torch.empty((4, 512, 256), device="cuda") for _ in range(2)]
        for w in dW:
            px.poetx_grouped_bwd_weight(desc, X, dZ, off, w, False)
        assert torch.equal(dW[0], dW[1]) and a.shape == (517, 512)


def test_grouped_on_another_stream(lib):
    """The calls run on the current stream, behind what it holds."""
    X = torch.zeros((512, 256), dtype=torch.bfloat16, device="cuda")
    W = torch.randn((2, 256, 256), device="cuda").bfloat16()
    Z = torch.empty((512, 256), dtype=torch.bfloat16, device="cuda")
    off = offsets_of([200, 312])
    desc = px.make_grouped_desc(256, 256, 2, 512, px.BF16)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        X.copy_(torch.randn((512, 256), device="cuda"))
        px.poetx_grouped_fwd(desc, X, W, off, Z)
        got = Z.clone()
    st.synchronize()
    px.poetx_grouped_fwd(desc, X, W, off, Z)
    assert torch.equal(got, Z) and float(Z.abs().max()) > 0


# ------------------------------------------------------------------------------------ order
@pytest.mark.parametrize("n,groups", [(0, 3), (1, 1), (1, 512), (8, 64), (63, 5), (64, 2), (1000, 7), (8192, 128), (8193, 128), (10000, 512), (131072, 100), (300001, 3)])
@pytest.mark.parametrize("dropped", [0.0, 0.3, 1.0])
def test_group_order(lib, n, groups, dropped):
    rng = np.random.default_rng(n + groups)
    ids = rng.integers(0, groups, n)
    if groups > 4:
        ids[ids == 3] = 2                          # a group without rows
    gone = rng.random(n) < dropped
    ids[gone] = rng.choice([-1, groups, groups + 5, -2 ** 31, 2 ** 31 - 1], n)[gone]
    keep = (ids >= 0) & (ids < groups)
    want_off = np.r_[0, np.cumsum(np.bincount(ids[keep], minlength=groups))]
    want = np.full(n, -1)
    kept = np.flatnonzero(keep)
    want[: len(kept)] = kept[np.argsort(ids[keep], kind="stable")]
    off = torch.full((groups + 1,), -7, dtype=torch.int32, device="cuda")
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, px.poetx_group_order_workspace_bytes(n, groups)),), 255, dtype=torch.uint8, device="cuda")
    px.poetx_group_order(torch.from_numpy(ids.astype(np.int32)).cuda(), off, order, ws)
    assert np.array_equal(off.cpu().numpy(), want_off) and np.array_equal(order.cpu().numpy(), want)


# ------------------------------------------------------------------------------------ sizes at which every kernel runs
def reference(kind, x, w, counts, dz=None):
    """float64 results and sums of magnitudes, group by group, on the GPU."""
    a, outs, mags = 0, [], []
    for g, c in enumerate(counts):
        if kind == "weight":
            l, r = dz[a: a + c].double().t(), x[a: a + c].double()
        else:
            l, r = x[a: a + c].double(), w[g].double().t() if kind == "fwd" else w[g].double()
        outs.append(l @ r)
        mags.append(l.abs() @ r.abs())
        a += c
    return (torch.stack if kind == "weight" else torch.cat)(outs), (torch.stack if kind == "weight" else torch.cat)(mags)


def within(got, ref, mag, K, dtype):
    lim = (K + 4) * 2.0 ** -24 * mag + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * ref.abs() + 1e-37
    return bool((torch.isfinite(got) & ((got.double() - ref).abs() <= lim)).all())


def spread(groups, rows, seed=0):
    """Uneven group sizes, some of them zero, that add up to `rows`."""
    rng = np.random.default_rng(seed)
    p = np.exp(rng.standard_normal(groups)) * (rng.random(groups) > 0.1)
    if p.sum() == 0:
        p[:] = 1
    return rng.multinomial(rows, p / p.sum()).tolist()


LARGE = [
    # groups, rows, d_in, d_out
    (1, 4096, 1024, 4096), (1, 2000, 1416, 2056), (8, 5000, 1032, 3000), (64, 6000, 520, 1376), (3, 1300, 1824, 1760), (5, 9000, 264, 776), (200, 3000, 256, 512),
    (300, 2000, 128, 136), (16, 8192, 512, 512), (2, 700, 2600, 96), (1, 333, 4000, 1000), (4, 12000, 40, 2048),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,rows,m,n", LARGE)
def test_grouped_large(lib, groups, rows, m, n, dtype):
    counts, dt = spread(groups, rows), DT[dtype]
    off = offsets_of(counts)
    g = torch.Generator(device="cuda").manual_seed(groups + rows)
    X, dZ = (torch.randn((rows, d), device="cuda", generator=g).to(dt) for d in (m, n))
    W = (torch.randn((groups, n, m), device="cuda", generator=g) * 0.02).to(dt)
    desc = px.make_grouped_desc(m, n, groups, rows, CODE[dtype])
    ws = torch.empty(max(256, px.poetx_grouped_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    Z, dX, dW = torch.empty((rows, n), dtype=dt, device="cuda"), torch.empty((rows, m), dtype=dt, device="cuda"), torch.empty((groups, n, m), device="cuda")
    px.poetx_grouped_fwd(desc, X, W, off, Z, ws)
    px.poetx_grouped_bwd_input(desc, dZ, W, off, dX, ws)
    px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, False, ws)
    assert within(Z, *reference("fwd", X, W, counts), m, dtype)
    assert within(dX, *reference("input", dZ, W, counts), n, dtype)
    ref, mag = reference("weight", X, None, counts, dZ)
    assert within(dW, ref, mag, rows, "f32")
    px.poetx_grouped_bwd_weight(desc, X, dZ, off, dW, True, ws)
    assert within(dW, 2 * ref, 2 * mag, rows, "f32")


@pytest.mark.parametrize("act", ["same", "mx4"])
@pytest.mark.parametrize("groups,rows,m,n", LARGE + [(1, 16, 2048, 8192), (1, 100, 1024, 4096), (1, 8, 512, 14336), (40, 1200, 384, 640), (1, 60, 4096, 6000), (64, 300, 256, 1376)])
def test_grouped_mx4_large(lib, groups, rows, m, n, act):
    counts = spread(groups, rows)
    off = offsets_of(counts)
    g = torch.Generator(device="cuda").manual_seed(groups + rows)
    X, dZ = (torch.randn((rows, d), device="cuda", generator=g).bfloat16() for d in (m, n))
    Q = quantised((torch.randn((groups * n, m), device="cuda", generator=g) * 0.02).bfloat16())
    W, Xr = torch.empty((groups * n, m), dtype=torch.bfloat16, device="cuda"), X
    px.poetx_mx4_dequantize(Q, W)
    if act == "mx4":
        Xr = torch.empty_like(X)
        px.poetx_mx4_dequantize(quantised(X), Xr)
    desc = px.make_grouped_desc(m, n, groups, rows, px.BF16, px.GROUPED_W_MX4 | (px.GROUPED_X_MX4 if act == "mx4" else 0))
    ws = torch.full((px.poetx_grouped_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    Z, dX = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, m), dtype=torch.bfloat16, device="cuda")
    px.poetx_grouped_fwd(desc, X, Q, off, Z, ws)
    px.poetx_grouped_bwd_input(desc, dZ, Q, off, dX, ws)
    W = W.view(groups, n, m)
    assert within(Z, *reference("fwd", Xr, W, counts), m, "bf16")
    assert within(dX, *reference("input", dZ, W, counts), n, "bf16")


@pytest.mark.parametrize("groups,rows,m,n,before,behind", [
    (1, 272, 136, 2056, 0, 0), (1, 300, 1416, 2056, 3, 130), (5, 700, 1032, 1000, 1, 0), (200, 5000, 264, 520, 0, 7), (300, 9000, 128, 136, 0, 0),      # tiles of 64 x 128
    (16, 8192, 512, 512, 0, 0), (2, 2100, 2056, 3000, 0, 5), (1, 1990, 1000, 2048, 9, 9),                                                              # 128 x 128
    (4, 5000, 2600, 2072, 2, 3), (8, 4096, 1000, 2056, 0, 0), (1, 2100, 2632, 2056, 65, 65),                                                           # 128 x 256
    (1, 219, 12040, 1152, 0, 0), (8, 106, 11848, 640, 7, 0), (3, 355, 10912, 1568, 0, 9), (1, 1474, 12544, 352, 2, 2)])                                # contractions in parts
def test_grouped_mx4_decoded_on_the_way(lib, groups, rows, m, n, before, behind):
    """More rows than a handful, with NaN in every row of X that no group has, between its rows and in the weight of a group without rows."""
    counts = spread(groups, rows)
    off = (offsets_of(counts) + before).int()
    g = torch.Generator(device="cuda").manual_seed(groups + rows + m)
    X, _ = strided(before + rows + behind, m, 24, torch.bfloat16, 8)
    X[before: before + rows] = torch.randn((rows, m), device="cuda", generator=g).bfloat16()
    values = (torch.randn((groups, n, m), device="cuda", generator=g) * 0.02).bfloat16()
    for k, c in enumerate(counts):
        if c == 0:
            values[k] = float("nan")
    Q = quantised(values.view(groups * n, m))
    W = torch.empty((groups * n, m), dtype=torch.bfloat16, device="cuda")
    px.poetx_mx4_dequantize(Q, W)
    desc = px.make_grouped_desc(m, n, groups, before + rows + behind, px.BF16, px.GROUPED_W_MX4)
    ws = torch.full((px.poetx_grouped_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    Z, flat = strided(before + rows + behind, n, 16, torch.bfloat16, 8, fill=3.0)
    px.poetx_grouped_fwd(desc, X, Q, off, Z, ws)
    assert within(Z[before: before + rows], *reference("fwd", X[before: before + rows], W.view(groups, n, m), counts), m, "bf16")
    again = torch.empty((before + rows + behind, n), dtype=torch.bfloat16, device="cuda")
    px.poetx_grouped_fwd(desc, X, Q, off, again, ws)
    assert torch.equal(again[before: before + rows], Z[before: before + rows])
    Z[before: before + rows] = 3.0
    assert bool((flat == 3.0).all()), "written where no group is"


def test_grouped_mx4_decoded_not_finite(lib):
    """An infinity or NaN of X stays in its row, one of the weight in its block's column of the groups that read it."""
    m, n, counts = 392, 2056, [130, 0, 400]
    G, rows = len(counts), sum(counts)
    g = torch.Generator(device="cuda").manual_seed(11)
    X = torch.randn((rows, m), device="cuda", generator=g).bfloat16()
    W = (torch.randn((G, n, m), device="cuda", generator=g) * 0.02).bfloat16()
    X[129, 391], X[130, 0], X[529, 128], W[2, 2055, 391], W[0, 0, 5] = float("nan"), float("inf"), float("-inf"), float("nan"), float("inf")
    desc = px.make_grouped_desc(m, n, G, rows, px.BF16, px.GROUPED_W_MX4)
    ws = torch.empty(px.poetx_grouped_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    Z = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    px.poetx_grouped_fwd(desc, X, quantised(W.view(G * n, m)), offsets_of(counts), Z, ws)
    want = torch.zeros_like(Z, dtype=torch.bool)
    want[129] = want[130] = want[529] = True
    want[130:, 2055] = want[:130, 0] = True
    assert torch.equal(~torch.isfinite(Z), want)


def test_grouped_mx4_decoded_past_32_bits(lib):
    """Rows of X and Z more than 2^32 bytes from the first."""
    m, n, rows, ld = 136, 2056, 2600, 1 << 21
    counts = [1100, 0, 1500]
    g = torch.Generator(device="cuda").manual_seed(5)
    X = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")[:, :m]
    Z = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")[:, :n]
    X.copy_(torch.randn((rows, m), device="cuda", generator=g).bfloat16())
    Q = quantised((torch.randn((3 * n, m), device="cuda", generator=g) * 0.02).bfloat16())
    W = torch.empty((3 * n, m), dtype=torch.bfloat16, device="cuda")
    px.poetx_mx4_dequantize(Q, W)
    desc = px.make_grouped_desc(m, n, 3, rows, px.BF16, px.GROUPED_W_MX4)
    ws = torch.empty(px.poetx_grouped_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    px.poetx_grouped_fwd(desc, X, Q, offsets_of(counts), Z, ws)
    assert within(Z, *reference("fwd", X, W.view(3, n, m), counts), m, "bf16")


@pytest.mark.parametrize("dtype,kind,m,n,counts,before,behind", [
    ("bf16", "fwd", 5568, 512, [637], 0, 0), ("bf16", "fwd", 7808, 1248, [200, 0, 300, 37, 251], 3, 9), ("bf16", "input", 1408, 5088, [221], 0, 70),
    ("bf16", "input", 776, 6368, [500, 607], 5, 0), ("f32", "fwd", 1760, 576, [1140], 0, 0), ("f32", "input", 516, 2692, [100, 0, 140], 2, 3)])
def test_grouped_split_contraction(lib, dtype, kind, m, n, counts, before, behind):
    """Few tiles and a long contraction: parts in the workspace, added by another launch, and the same without one."""
    rows, dt = before + sum(counts) + behind, DT[dtype]
    off = (offsets_of(counts) + before).int()
    g = torch.Generator(device="cuda").manual_seed(m)
    d_in, d_out = (m, n) if kind == "fwd" else (n, m)
    x = torch.full((rows, d_in), float("nan"), device="cuda", dtype=dt)
    x[before: before + sum(counts)] = torch.randn((sum(counts), d_in), device="cuda", generator=g).to(dt)
    W = (torch.randn((len(counts), n, m), device="cuda", generator=g) * 0.02).to(dt)
    desc = px.make_grouped_desc(m, n, len(counts), rows, CODE[dtype])
    need = px.poetx_grouped_workspace_bytes(desc)
    assert need >= 2 * rows * d_out * 4
    ref, mag = reference(kind, x[before:], W, counts)
    call = px.poetx_grouped_fwd if kind == "fwd" else px.poetx_grouped_bwd_input
    for ws in (torch.full((need // 4,), float("nan"), device="cuda").view(torch.uint8), None):
        out, flat = strided(rows, d_out, 16, dt, fill=3.0)
        call(desc, x, W, off, out, ws)
        assert within(out[before: before + sum(counts)], ref, mag, d_in, dtype)
        out[before: before + sum(counts)] = 3.0
        assert bool((flat == 3.0).all()), "written where no group is"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_grouped_offsets_past_32_bits(lib, dtype):
    """Rows further apart than 2^31 elements (and 2^32 bytes) from the first one."""
    ld, rows, m, n = 1 << 15, 70000, 64, 128
    flat = torch.empty(rows * ld, dtype=DT[dtype], device="cuda")
    X = flat.view(rows, ld)[:, :m]
    tail = 300
    X[-tail:] = torch.randn((tail, m), device="cuda").to(DT[dtype])
    W = torch.randn((3, n, m), device="cuda").to(DT[dtype])
    off = torch.tensor([rows - tail, rows - 200, rows - 200, rows], dtype=torch.int32, device="cuda")
    Z = flat.view(rows, ld)[:, 1024: 1024 + n]      # the span of the output overlaps the input's: refused
    desc = px.make_grouped_desc(m, n, 3, rows, CODE[dtype])
    with pytest.raises(px.PoetxError):
        px.poetx_grouped_fwd(desc, X, W, off, Z)
    Z = torch.zeros((rows, n), dtype=DT[dtype], device="cuda")
    px.poetx_grouped_fwd(desc, X, W, off, Z)
    counts = [100, 0, 200]
    assert within(Z[-tail:], *reference("fwd", X[-tail:], W, counts), m, dtype) and not bool(Z[:-tail].any())
    dW = torch.empty((3, n, m), device="cuda")
    px.poetx_grouped_bwd_weight(desc, X, Z, off, dW, False)
    assert within(dW, *reference("weight", X[-tail:], None, counts, Z[-tail:]), tail, "f32")
    dX = flat.view(rows, ld)[:, 2048: 2048 + m]
    px.poetx_grouped_bwd_input(desc, Z, W, off, dX)
    assert within(dX[-tail:], *reference("input", Z[-tail:], W, counts), n, dtype)
    if dtype == "bf16":
        Q = quantised(X[-tail:])
        rows_q = (1 << 32) // 4096 + 3                  # more than 2^32 codes
        big = torch.zeros((rows_q, 4096), dtype=torch.bfloat16, device="cuda")
        big[-tail:, :m] = X[-tail:]
        Qb = quantised(big)
        del big
        back = torch.empty((rows_q, 4096), dtype=torch.bfloat16, device="cuda")
        px.poetx_mx4_dequantize(Qb, back)
        want = torch.empty((tail, m), dtype=torch.bfloat16, device="cuda")
        px.poetx_mx4_dequantize(Q, want)
        assert torch.equal(back[-tail:, :m], want) and not bool(back[-1, m:].any())


@pytest.mark.parametrize("weight", ["dense", "mx4", "both"])
def test_grouped_in_a_graph(lib, weight):
    """Captured once, replayed with other rows, offsets and ids in the same buffers."""
    m, n, groups, tokens, k = 256, 384, 6, 500, 2
    rows = tokens * k
    g = torch.Generator(device="cuda").manual_seed(2)
    W = (torch.randn((groups, n, m), device="cuda", generator=g) * 0.05).bfloat16()
    Wx = W if weight == "dense" else quantised(W.view(groups * n, m))
    desc = px.make_grouped_desc(m, n, groups, rows, px.BF16, {"dense": 0, "mx4": px.GROUPED_W_MX4, "both": px.GROUPED_W_MX4 | px.GROUPED_X_MX4}[weight])
    ws = torch.empty(max(256, px.poetx_grouped_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    ows = torch.empty(max(256, px.poetx_group_order_workspace_bytes(rows, groups)), dtype=torch.uint8, device="cuda")
    ids, x = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros((rows, m), dtype=torch.bfloat16, device="cuda")
    off, order = torch.zeros(groups + 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    Z, dX = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda"), torch.zeros((rows, m), dtype=torch.bfloat16, device="cuda")

    def calls():
        px.poetx_group_order(ids, off, order, ows)
        px.poetx_grouped_fwd(desc, x, Wx, off, Z, ws)
        px.poetx_grouped_bwd_input(desc, Z, Wx, off, dX, ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        ids.copy_(torch.randint(0, groups, (rows,), device="cuda", generator=g).int())
        x.copy_(torch.randn((rows, m), device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (off, order, Z, dX)]
        for t in (off, order, Z, dX):
            t.zero_()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (off, order, Z, dX))) and float(dX.abs().max()) > 0


def test_experts_example(lib):
    """The example layer in fp32 against torch autograd in float64, and its 4-bit forms' command line."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "experts.py")
    spec = importlib.util.spec_from_file_location("experts_example", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    tokens, d, f, E, k = 50, 64, 96, 5, 2
    gen = torch.Generator(device="cuda").manual_seed(4)
    W1, W2 = (torch.stack([ex.merged(torch.randn(s, device="cuda", generator=gen) * 0.1, 16, 3, 0.02, gen) for _ in range(E)]) for s in ((f, d), (d, f)))
    x, dout = (torch.randn((tokens, d), device="cuda", generator=gen) for _ in range(2))
    ids = torch.randint(-1, E, (tokens, k), device="cuda", generator=gen)
    gates = torch.rand((tokens, k), device="cuda", generator=gen)
    layer = ex.Experts(W1, W2, tokens, k)
    out = layer.forward(x, ids, gates)
    dx, dgate, (dW1, dW2) = layer.backward(dout, weights=True)
    leaves = [t.double().requires_grad_() for t in (x, gates, W1, W2)]
    xr, gr, W1r, W2r = leaves
    e = ids.clamp(min=0)
    h = torch.einsum("tkfd,td->tkf", W1r[e], xr).clamp(min=0) ** 2
    ref = (torch.einsum("tkdf,tkf->tkd", W2r[e], h) * (gr * (ids >= 0)).unsqueeze(2)).sum(1)
    ref.backward(dout.double())
    for got, want in ((out, ref), (dx, xr.grad), (dgate, gr.grad), (dW1, W1r.grad), (dW2, W2r.grad)):
        assert float((got.double() - want.detach()).abs().max()) <= 1e-5 * float(want.detach().abs().max())
    small = ["--tokens", "70", "--experts", "4", "--d", "256", "--hidden", "192", "--block", "64", "--steps", "1"]
    for more in ([], ["--activations", "mx4"], ["--weights", "dense"]):
        assert ex.main(small + more) == 0
