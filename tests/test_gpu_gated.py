"""8-bit buffers, the gated feed-forward block, its backward pass and the weight gradient that reads 8-bit rows, against plain float64 forms written here.

Bounds, per element, with u = 2^-24 (half a step of fp32) and r the half step of the result's type (2^-8 bf16, u fp32):
  G, U     products of two bf16 (or of a bf16 and a 4-bit value) are exact in fp32, so a sum of K of them is off by at most eG = (K + 2) u sum |x w| (fp32: a rounding
           more per product, within the same), kept ones by r |G| more.
  s        z is rounded up to 5 times and multiplied by a rounded log2(e): the exponent is off by 7 u |z|; exp, the sum and the reciprocal by 2u, u, 2u of themselves.  What
           reaches s = 1 / (1 + e^-z) of an error of e^-z is its share 1 - s:      es = (1 - s) (7 |z| + 2) u + 3 u, relative.
  act      g s: relative es + u, and act' is at most 1.13 in size for either activation:      ea = |act| (es + u) + 1.13 eG.
  act'     s (1 + Q (1 - s)), Q = g z': 1 - s is off by s es + u, Q by 5 u, the rest by 3 roundings, and act'' is at most 1:
           ed = s |Q| ((1 - s) 5 u + s es + u) + |act'| (es + 3 u) + s u + eG.
           From z = 20 on 1 + e^-z rounds to 1, so that 1 - s is 0 and what is lost is Q (1 - s).
           s below 2^-126 may be taken as 0: 2^-126 times g or Q (under 300 where that is so), less than 1e-35.
  H        |act| eU + |U| ea + ea eU + 2 u |H|, rounded: + r |H|;  dU = dH act, dG = dH U act' likewise.
  dW       as the grouped products', values of 8-bit codes being exact.
A value of 8 bits is off by at most 2^-6 2^e, 2^e being the power of two at or below the largest of its block (half of that unless it is clamped), and by what moved it before."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_grouped import CODE, DT, oracle_values, quantised, split_buffer, strided

pytestmark = pytest.mark.gpu

U24 = 2.0 ** -24
ACT = {"silu": px.GATED_SILU, "gelu": px.GATED_GELU}


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U24


def host(t):
    return t.detach().double().cpu()


def scratch(nbytes):
    """A workspace that holds NaN."""
    return torch.full((nbytes // 4 + 64,), float("nan"), device="cuda").view(torch.uint8) if nbytes else None


# ------------------------------------------------------------------------------------ eight bits
def oracle_mx8(x):
    """float64 [rows][cols] -> codes [rows][mp], scale bytes [rows][mp / 32], by the definition."""
    rows, cols = x.shape
    mp = -(-cols // 128) * 128
    p = np.zeros((rows, mp))
    p[:, :cols] = x
    p = p.reshape(rows, mp // 32, 32)
    with np.errstate(all="ignore"):
        top = np.abs(p).max(-1)
        scale = np.where(top > 0, np.clip(np.frexp(top)[1] - 1 + 127, 0, 254), 0)
        bad = ~np.isfinite(p).all(-1)
        code = np.clip(np.rint(np.ldexp(p, 133 - scale[..., None])), -127, 127)
    return np.where(bad[..., None], 0, code).astype(np.int64).reshape(rows, mp), np.where(bad, 255, scale)


def mx8_values(code, scale, cols):
    with np.errstate(over="ignore"):
        v = np.ldexp(code.reshape(*scale.shape, 32).astype(float), (scale - 133)[..., None])
    return np.where((scale == 255)[..., None], np.nan, v).reshape(code.shape)[:, :cols]


def split_mx8(Q, rows, cols):
    q = Q.cpu().numpy()
    mp = -(-cols // 128) * 128
    off = -(-rows * mp // 256) * 256
    return q[: rows * mp].view(np.int8).reshape(rows, mp).astype(np.int64), q[off: off + rows * mp // 32].reshape(rows, mp // 32).astype(np.int64)


def mx8_of(X, fill=255):
    """X (rows x cols on the device) -> its 8-bit buffer, which held `fill` before."""
    Q = torch.full((px.poetx_mx8_bytes(*X.shape),), fill, dtype=torch.uint8, device="cuda")
    px.poetx_mx8_quantize(X, Q)
    return Q


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 0), (2, 33, 7, 1), (4, 127, 1, 3), (7, 128, 8, 0), (17, 160, 0, 0),
                                                 (33, 257, 3, 1), (9, 1376, 0, 0), (1, 4096, 0, 0), (300, 520, 8, 8)])
def test_mx8_round_trip(lib, rows, cols, pad, shift, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-30, 30, (rows, 1)).astype(float))
    X, _ = strided(rows, cols, pad, DT[dtype], shift)
    X.copy_(torch.from_numpy(x).to(DT[dtype]))
    code, scale = oracle_mx8(host(X).numpy())
    Q = mx8_of(X)
    got_c, got_s = split_mx8(Q, rows, cols)
    assert np.array_equal(got_s, scale) and np.array_equal(got_c, code)
    want = mx8_values(code, scale, cols)
    for out_type in ("bf16", "f32"):
        out, flat = strided(rows, cols, pad, DT[out_type], shift, fill=7.0)
        px.poetx_mx8_dequantize(Q, out)
        assert np.array_equal(host(out).numpy(), want)
        out.fill_(7.0)
        assert bool((flat == 7.0).all()), "written outside the matrix"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mx8_ties_and_extremes(lib, dtype):
    """Ties, what is clamped, zeros, the smallest and largest numbers, infinities and NaN."""
    half = np.arange(16) + 0.5
    rows = [np.r_[64.0, half, -half[:15]], np.r_[127.5, 127.25, -127.5, 126.5, 125.5, np.arange(27) * 4.5], np.r_[1.0, half * 2.0 ** -6, -half[:15] * 2.0 ** -6],
            np.zeros(32), np.full(32, -0.0), np.full(32, 2.0 ** -126), np.full(32, 2.0 ** -130), np.full(32, 3.0e38), np.arange(32) * 2.0 ** -133,
            np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.ones(7), np.nan, np.zeros(24)], np.r_[1e30, np.full(31, 1e-30)], np.full(32, 255.0)]
    X = torch.from_numpy(np.array(rows)).to(DT[dtype]).cuda()
    code, scale = oracle_mx8(host(X).numpy())
    Q = mx8_of(X)
    got_c, got_s = split_mx8(Q, *X.shape)
    assert np.array_equal(got_s, scale) and np.array_equal(got_c, code)
    out = torch.empty_like(X)
    px.poetx_mx8_dequantize(Q, out)
    assert np.array_equal(host(out).numpy(), mx8_values(code, scale, 32), equal_nan=True)


def test_mx8_all_codes_and_scales(lib):
    """A buffer a caller built: every code under every scale byte, -128 and NaN among them; what bf16 or fp32 cannot hold is infinite."""
    code = np.tile(np.arange(-128, 128), (256, 1))
    scale = np.tile(np.arange(256)[:, None], (1, 8))
    Q = torch.from_numpy(np.concatenate([code.astype(np.int8).view(np.uint8).ravel(), scale.astype(np.uint8).ravel()])).cuda()
    want = torch.from_numpy(mx8_values(code, scale, 256))
    for dtype in DT.values():
        out = torch.empty((256, 256), dtype=dtype, device="cuda")
        px.poetx_mx8_dequantize(Q, out)
        assert np.array_equal(host(out).numpy(), want.to(dtype).double().numpy(), equal_nan=True)


# ------------------------------------------------------------------------------------ the block
def activation(act, G, eG):
    """act, act' and the bounds of their errors for G known to eG."""
    if act == "silu":
        z, Q = G, G
    else:
        c = 2 * math.sqrt(2 / math.pi)
        z, Q = c * (G + 0.044715 * G ** 3), G * c * (1 + 3 * 0.044715 * G ** 2)
    s, rest = torch.sigmoid(z), torch.sigmoid(-z)
    es = rest * (7 * z.abs() + 2) * U24 + 3 * U24
    a, d = G * s, s * (1 + Q * rest)
    ea = a.abs() * (es + U24) + 1.13 * eG + 1e-35
    ed = s * Q.abs() * (rest * 5 * U24 + s * es + U24) + d.abs() * (es + 3 * U24) + s * U24
    ed = torch.where(z > 20, Q.abs() * rest + 4 * U24, ed)
    return a, d, ea, ed + eG + 1e-35


def near(got, ref, lim, what):
    assert bool(torch.isfinite(got).all()), what
    err = (got - ref).abs()
    assert bool((err <= lim + 1e-36).all()), (what, float(err.max()), float((err / (lim + 1e-36)).max()))


def forward_of(act, G, U, eG, eU, r):
    a, _, ea, _ = activation(act, G, eG)
    H = a * U
    return H, a.abs() * eU + U.abs() * ea + ea * eU + (2 * U24 + 2 * r) * H.abs()


def backward_of(act, dH, G, U, eG, eU, r):
    a, d, ea, ed = activation(act, G, eG)
    dG, dU = dH * U * d, dH * a
    edG = dH.abs() * ((U.abs() + eU) * ed + d.abs() * eU) + (2 * U24 + 2 * r) * dG.abs()
    return dG, dU, edG, dH.abs() * ea + (U24 + 2 * r) * dU.abs()


class Block:
    """Inputs of a block over groups of `counts` rows, with `before` rows ahead of them and `extra` behind that no group has (NaN), and G, U in 64 bits."""

    def __init__(self, counts, m, n, dtype, act="silu", weight="dense", pads=(0, 0), shift=0, before=0, extra=0, seed=0):
        rng = np.random.default_rng(seed + m + 7 * n + 31 * len(counts))
        self.m, self.n, self.act, self.dtype, self.dt = m, n, act, dtype, DT[dtype]
        self.pads, self.shift = pads, shift
        self.groups, self.rows, self.a, self.b = len(counts), before + sum(counts) + extra, before, before + sum(counts)
        ends = before + np.r_[0, np.cumsum(counts)]
        self.off = torch.tensor(ends, dtype=torch.int32, device="cuda")
        live = slice(self.a, self.b)
        self.X, _ = strided(self.rows, m, pads[0], self.dt, shift)
        self.dH, _ = strided(self.rows, n, pads[1], self.dt, shift)
        self.X[live].copy_(torch.from_numpy(rng.standard_normal((sum(counts), m))).to(self.dt))
        self.dH[live].copy_(torch.from_numpy(rng.standard_normal((sum(counts), n)) * 0.1).to(self.dt))
        W = torch.from_numpy(rng.standard_normal((self.groups, 2 * n, m)) * 1.5 / m ** 0.5).to(self.dt).cuda()
        self.flags, self.W, Wh = 0, W, host(W)
        if weight == "mx4":
            self.flags, self.W = px.GATED_W_MX4, quantised(W.view(-1, m))
            Wh = torch.from_numpy(oracle_values(*split_buffer(self.W, self.groups * 2 * n, m), m)).view(self.groups, 2 * n, m)
        x = host(self.X)
        self.Wh, self.xh = Wh, x
        GU, mag = torch.zeros((self.rows, 2 * n), dtype=torch.float64), torch.zeros((self.rows, 2 * n), dtype=torch.float64)
        for g in range(self.groups):
            p, q = int(ends[g]), int(ends[g + 1])
            GU[p:q], mag[p:q] = x[p:q] @ Wh[g].t(), x[p:q].abs() @ Wh[g].abs().t()
        e = (m + 2) * U24 * mag
        self.G, self.U, self.eG, self.eU = GU[live, :n], GU[live, n:], e[live, :n], e[live, n:]
        self.r = half_step(dtype)

    def desc(self, flags=0):
        return px.make_gated_desc(self.m, self.n, self.groups, self.rows, CODE[self.dtype], ACT[self.act], self.flags | flags)

    def ws(self, desc):
        return scratch(px.poetx_gated_workspace_bytes(desc))

    def out(self, pair=False):
        """An output of n columns or, as a pair, the halves of one of 2n; filled with 3, and what checks and refills it."""
        t, flat = strided(self.rows, self.n * (2 if pair else 1), self.pads[1], self.dt, self.shift, fill=3.0)
        return (t[:, : self.n], t[:, self.n:], flat) if pair else (t, flat)

    def untouched(self, what, flat, *tensors):
        """The live rows are the calls' own: what they hold is taken out, and everything else has to be 3."""
        kept = [t[self.a: self.b].clone() for t in tensors]
        for t in tensors:
            t[self.a: self.b] = 3.0
        assert bool((flat == 3.0).all()), what + ": written outside the rows"
        for t, k in zip(tensors, kept):
            t[self.a: self.b] = k

    def live(self, t):
        return host(t[self.a: self.b])


def run_forward(b):
    desc = b.desc()
    ws = b.ws(desc)
    H, flat = b.out()
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, ws=ws)
    ref, lim = forward_of(b.act, b.G, b.U, b.eG, b.eU, b.r / 2)
    near(b.live(H), ref, lim, "H")
    b.untouched("H", flat, H)
    H2, flat = b.out()
    G, U, flat2 = b.out(pair=True)
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H2, G, U, ws=b.ws(desc))
    assert torch.equal(H2[b.a: b.b], H[b.a: b.b]), "H with and without what is kept"
    near(b.live(G), b.G, b.eG + b.r * (b.G.abs() + b.eG), "G kept")
    near(b.live(U), b.U, b.eU + b.r * (b.U.abs() + b.eU), "U kept")
    b.untouched("H", flat, H2)
    b.untouched("G, U", flat2, G, U)
    return H, G, U


def run_forward_mx8(b):
    """Kept in eight bits: codes of the rows that some group has, and those of no group as they were."""
    desc = b.desc(px.GATED_HELD_MX8)
    H, flat = b.out()
    size = px.poetx_mx8_bytes(b.rows, b.n)
    QG, QU = (torch.full((size,), 77, dtype=torch.uint8, device="cuda") for _ in range(2))
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, QG, QU, ws=b.ws(desc))
    ref, lim = forward_of(b.act, b.G, b.U, b.eG, b.eU, b.r / 2)
    near(b.live(H), ref, lim, "H")
    b.untouched("H", flat, H)
    values = []
    for Q, v, e in ((QG, b.G, b.eG), (QU, b.U, b.eU)):
        code, scale = split_mx8(Q, b.rows, b.n)
        for c in (code, scale):
            assert (np.delete(c, np.arange(b.a, b.b), 0) == 77).all(), "rows of no group"
        code, scale = code[b.a: b.b], scale[b.a: b.b]
        assert (code[:, b.n:] == 0).all() and (scale[:, -(-b.n // 32):] == 0).all(), "past the columns"
        got = torch.from_numpy(mx8_values(code, scale, b.n))
        wide = torch.nn.functional.pad((v.abs() + e), (0, -b.n % 32)).view(len(v), -(-b.n // 32), 32)
        top = torch.repeat_interleave(wide.amax(-1), 32, 1)[:, : b.n]
        near(got, v, e + 2.0 ** -6 * torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300)))), "kept in eight bits")
        # and each block's codes reach up to its scale, as quantising its own values gives
        again = oracle_mx8(got.numpy())
        assert ((again[1] == scale[:, : again[1].shape[1]]) | (again[0].reshape(*again[1].shape, 32) == 0).all(-1)).all()
        values.append(got)
    return QG, QU, values


def run_backward(b, held):
    """From what is kept: G and U of the bound's formulas are the kept values themselves."""
    if held == "mx8":
        QG, QU, (G, U) = run_forward_mx8(b)
        desc = b.desc(px.GATED_HELD_MX8)
    else:
        _, QG, QU = run_forward(b)
        G, U = b.live(QG), b.live(QU)
        desc = b.desc()
    dG, dU, flat = b.out(pair=True)
    H, flat2 = b.out()
    px.poetx_gated_bwd(desc, b.dH, QG, QU, b.off, dG, dU, H)
    zero = torch.zeros_like(G)
    rG, rU, lG, lU = backward_of(b.act, b.live(b.dH), G, U, zero, zero, b.r / 2)
    near(b.live(dG), rG, lG, "dG")
    near(b.live(dU), rU, lU, "dU")
    rH, lH = forward_of(b.act, G, U, zero, zero, b.r / 2)
    near(b.live(H), rH, lH, "H again")
    b.untouched("dG, dU", flat, dG, dU)
    b.untouched("H again", flat2, H)
    eG, eU, flat = b.out(pair=True)
    px.poetx_gated_bwd(desc, b.dH, QG, QU, b.off, eG, eU)
    assert torch.equal(eG, dG) and torch.equal(eU, dU), "without H"
    return dG, dU


def run_recompute(b):
    desc = b.desc()
    dG, dU, flat = b.out(pair=True)
    H, flat2 = b.out()
    px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, dG, dU, H, ws=b.ws(desc))
    rG, rU, lG, lU = backward_of(b.act, b.live(b.dH), b.G, b.U, b.eG, b.eU, b.r / 2)
    near(b.live(dG), rG, lG, "dG")
    near(b.live(dU), rU, lU, "dU")
    rH, lH = forward_of(b.act, b.G, b.U, b.eG, b.eU, b.r / 2)
    near(b.live(H), rH, lH, "H again")
    b.untouched("dG, dU", flat, dG, dU)
    b.untouched("H again", flat2, H)
    eG, eU, _ = b.out(pair=True)
    px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, eG, eU, ws=b.ws(desc))
    assert torch.equal(eG, dG) and torch.equal(eU, dU), "without H"


def run_all(*a, **k):
    b = Block(*a, **k)
    run_backward(b, "same")
    run_backward(b, "mx8")
    run_recompute(b)


SHAPES = [
    # counts, m, n
    ([1], 1, 1), ([0], 8, 8), ([3], 7, 5), ([1, 0, 2], 33, 17), ([5, 1, 0, 130, 64], 64, 96), ([31, 33, 32], 100, 60),
    ([0, 0, 7], 256, 128), ([257], 130, 258), ([128, 129, 127], 128, 256), ([300, 0, 1, 211], 256, 320), ([64] * 5, 96, 1376),
    ([1] * 70, 64, 64), ([2, 0] * 70, 40, 72), ([600, 5], 512, 264), ([1], 4096, 520), ([16], 640, 256), ([260, 255], 1408, 136), ([70], 2048, 40),
]


@pytest.mark.parametrize("dtype,act", [("bf16", "silu"), ("f32", "gelu")])
@pytest.mark.parametrize("counts,m,n", SHAPES)
def test_gated(lib, counts, m, n, dtype, act):
    run_all(counts, m, n, dtype, act)


@pytest.mark.parametrize("dtype,act", [("bf16", "gelu"), ("f32", "silu")])
@pytest.mark.parametrize("pads,shift,before,extra", [((8, 16), 0, 0, 0), ((3, 5), 0, 2, 9), ((0, 0), 1, 0, 0), ((8, 8), 8, 70, 130), ((1, 0), 3, 0, 1)])
def test_gated_strides(lib, pads, shift, before, extra, dtype, act):
    run_all([17, 0, 150, 3], 136, 200, dtype, act, pads=pads, shift=shift, before=before, extra=extra)


@pytest.mark.parametrize("counts,m,n", SHAPES + [([17, 40], 2048, 264), ([513], 1408, 512), ([1, 1, 0, 1], 1024, 1376)])
def test_gated_mx4(lib, counts, m, n):
    run_all(counts, m, n, "bf16", weight="mx4")


@pytest.mark.parametrize("pads,shift,before,extra", [((8, 16), 0, 0, 0), ((3, 5), 0, 2, 9), ((0, 0), 1, 0, 0), ((8, 8), 8, 70, 130)])
def test_gated_mx4_strides(lib, pads, shift, before, extra):
    run_all([17, 0, 150, 3], 136, 200, "bf16", weight="mx4", pads=pads, shift=shift, before=before, extra=extra)


# Enough tiles for the streams, and contractions for them to be split, of whole vectors and of others.
LARGE = [
    # counts, m, n, pads (of X, of the rest)
    ([4096], 256, 2048, (0, 0)), ([4095], 264, 2047, (8, 3)), ([2048, 0, 2040], 136, 1030, (0, 0)), ([1000, 24], 320, 1280, (0, 8)), ([1023], 512, 1022, (0, 1)),
    ([130] * 9, 192, 257, (0, 0)), ([700, 0, 333], 2048, 72, (0, 0)), ([515], 4096, 66, (0, 0)), ([300], 3336, 129, (0, 0)), ([90] * 24, 128, 384, (0, 0)),
]


@pytest.mark.parametrize("dtype,act,weight", [("bf16", "gelu", "dense"), ("bf16", "silu", "mx4"), ("f32", "silu", "dense")])
@pytest.mark.parametrize("counts,m,n,pads", LARGE)
def test_gated_large(lib, counts, m, n, pads, dtype, act, weight):
    run_all(counts, m, n, dtype, act, weight, pads=pads, before=3, extra=5)


# One for every kernel that these lists do not reach, 8 more rows than the groups have counting: tiles of 256 x 256 and 128 x 128 and contractions in ranges, of whole vectors and not; a 4-bit
# weight decoded in ranges, on the largest tile, for a handful of rows, and written out first; fp32 tiles of 128 x 128.
PATHS = [
    ([2992], 136, 2056, "bf16", "dense"), ([2992], 520, 520, "bf16", "dense"), ([5992], 136, 1001, "bf16", "dense"), ([2000, 80, 2000], 136, 1032, "bf16", "dense"),
    ([92], 4104, 1032, "bf16", "dense"), ([192], 2056, 2100, "bf16", "dense"), ([1000, 1040], 4104, 66, "bf16", "dense"), ([292], 65, 1001, "bf16", "dense"),
    ([32], 4104, 2056, "bf16", "mx4"), ([1092, 1900], 6152, 130, "bf16", "mx4"), ([3000, 0, 2992], 264, 1001, "bf16", "mx4"), ([120], 65, 8192, "bf16", "mx4"),
    ([8], 64, 6200, "bf16", "mx4"), ([5992], 136, 2056, "bf16", "mx4"), ([1500, 1492], 65, 130, "bf16", "mx4"),
    ([2040], 1001, 1000, "bf16", "dense"), ([700, 0, 800], 1001, 515, "bf16", "dense"), ([1492], 916, 1032, "bf16", "mx4"), ([290], 3366, 416, "bf16", "mx4"), ([1397], 1014, 544, "f32", "dense"),
    ([20] * 300, 72, 40, "bf16", "dense"), ([20] * 300, 72, 40, "bf16", "mx4"), ([5] * 300, 72, 264, "f32", "dense"),
    ([1492], 2056, 2100, "f32", "dense"), ([700, 1348], 2056, 72, "f32", "dense"), ([292], 1032, 1032, "f32", "dense"), ([2992], 65, 130, "f32", "dense"),
]


@pytest.mark.parametrize("counts,m,n,dtype,weight", PATHS)
def test_gated_on_every_kernel(lib, counts, m, n, dtype, weight):
    run_all(counts, m, n, dtype, "silu" if n % 2 else "gelu", weight, before=3, extra=5)


@pytest.mark.parametrize("held", ["same", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_everywhere(lib, act, dtype, held):
    """Every size of G from far below to far above what the activations bend at, U and dH of ordinary size."""
    g = np.concatenate([np.linspace(-30, 30, 1021), np.geomspace(1e-30, 3e30, 300), -np.geomspace(1e-30, 3e30, 300), [0.0, -0.0]])
    n, rows, dt = 64, len(g), DT[dtype]
    G = torch.from_numpy(np.repeat(g[:, None], n, 1)).to(dt).cuda()      # a block of eight bits holds one size
    rng = np.random.default_rng(5)
    U, dH = (torch.from_numpy(rng.standard_normal((rows, n))).to(dt).cuda() for _ in range(2))
    QG, QU = (mx8_of(G), mx8_of(U)) if held == "mx8" else (G, U)
    if held == "mx8":
        G, U = G.clone(), U.clone()
        px.poetx_mx8_dequantize(QG, G)
        px.poetx_mx8_dequantize(QU, U)
    desc = px.make_gated_desc(8, n, 1, rows, CODE[dtype], ACT[act], px.GATED_HELD_MX8 if held == "mx8" else 0)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    dG, dU, H = (torch.empty((rows, n), dtype=dt, device="cuda") for _ in range(3))
    px.poetx_gated_bwd(desc, dH, QG, QU, off, dG, dU, H)
    zero = torch.zeros((rows, n), dtype=torch.float64)
    r = half_step(dtype)
    rG, rU, lG, lU = backward_of(act, host(dH), host(G).clamp(-1e6, 1e6), host(U), zero, zero, r / 2)      # the derivative: 0 or 1 long before
    near(host(dG), rG, lG, "dG")
    _, rU, _, lU = backward_of(act, host(dH), host(G), host(U), zero, zero, r / 2)
    near(host(dU), rU, lU, "dU")
    rH, lH = forward_of(act, host(G), host(U), zero, zero, r / 2)
    near(host(H), rH, lH, "H")


def test_gated_not_finite(lib):
    """NaN or an infinity of a row, of a group's weight or of what was kept stays in the elements that read it."""
    m, n, counts = 256, 128, [130, 70, 0, 300]
    b = Block(counts, m, n, "bf16")
    b.X[129, 255] = float("nan")
    b.W[2] = float("nan")                       # the weight of a group without rows
    b.W[3, 5, 7] = float("nan")                 # gate
    b.W[3, n + 9, 0] = float("inf")             # up
    want = torch.zeros((500, n), dtype=torch.bool, device="cuda")
    want[129] = want[200:, 5] = want[200:, 9] = True
    desc, mx8 = b.desc(), b.desc(px.GATED_HELD_MX8)
    H, dG, dU = (torch.empty((500, n), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, ws=b.ws(desc))
    assert torch.equal(~torch.isfinite(H), want)
    b.dH[17, 3] = float("inf")
    px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, dG, dU, ws=b.ws(desc))
    w = want.clone()
    w[17, 3] = True
    assert torch.equal(~torch.isfinite(dG), w)
    w[200:, 9] = False                          # dU does without U
    assert torch.equal(~torch.isfinite(dU), w)
    QG, QU = (torch.zeros(px.poetx_mx8_bytes(500, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    px.poetx_gated_fwd(mx8, b.X, b.W, b.off, H, QG, QU, ws=b.ws(mx8))
    assert torch.equal(~torch.isfinite(H), want)
    px.poetx_gated_bwd(mx8, b.dH, QG, QU, b.off, dG, dU, H)
    w = want.clone()
    w[200:, :32] = True                         # a block shares its NaN
    assert torch.equal(~torch.isfinite(H), w)
    w[17, 3] = True
    assert torch.equal(~torch.isfinite(dG), w)
    G = torch.tensor([[float("inf"), -float("inf"), float("nan"), 1.0] * 8], dtype=torch.bfloat16, device="cuda")
    one = torch.ones_like(G)
    d = px.make_gated_desc(8, 32, 1, 1, px.BF16)
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    dG, dU, H = (torch.empty_like(G) for _ in range(3))
    px.poetx_gated_bwd(d, one, G, one, off, dG, dU, H)
    for t, limits in ((H, (math.inf, 0.0)), (dU, (math.inf, 0.0)), (dG, (1.0, 0.0))):      # the activation's limits
        assert t[0, 0] == limits[0] and t[0, 1] == limits[1] and bool(torch.isnan(t[0, 2])) and bool(torch.isfinite(t[0, 3]))


def test_gated_offsets_out_of_range(lib):
    """Offsets past the rows, below zero or descending: no row has two results, nothing outside is touched."""
    m, n, rows = 128, 64, 100
    b = Block([rows], m, n, "bf16")
    off = torch.tensor([-5, 40, 30, 70, 1000], dtype=torch.int32, device="cuda")
    W = torch.cat([b.W * s for s in (1.0, 2.0, 0.5, 1.0)])
    for mode in ("fwd", "mx8", "again"):
        desc = px.make_gated_desc(m, n, 4, rows, px.BF16, px.GATED_SILU, px.GATED_HELD_MX8 if mode == "mx8" else 0)
        flat = torch.full((rows + 64, n), 3.0, dtype=torch.bfloat16, device="cuda")
        H, ws = flat[:rows], scratch(px.poetx_gated_workspace_bytes(desc))
        if mode == "again":
            dG, dU = (torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            px.poetx_gated_bwd_recompute(desc, b.dH, b.X, W, off, dG, dU, H, ws=ws)
        else:
            Q = [torch.zeros(px.poetx_mx8_bytes(rows, n), dtype=torch.uint8, device="cuda") for _ in range(2)] if mode == "mx8" else [None, None]
            px.poetx_gated_fwd(desc, b.X, W, off, H, *Q, ws=ws)
        for a, e, s in ((0, 40, 1.0), (40, 70, 0.5), (70, 100, 1.0)):
            ref, lim = forward_of("silu", b.G[a:e] * s, b.U[a:e] * s, b.eG[a:e], b.eU[a:e], b.r / 2)
            near(host(H[a:e]), ref, lim, (mode, a))
        assert bool((flat[rows:] == 3.0).all())


# ------------------------------------------------------------------------------------ the weight gradient of 8-bit rows
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,m,n,before,extra", [([1], 1, 1, 0, 0), ([0], 8, 8, 0, 0), ([3], 7, 5, 1, 2), ([5, 1, 0, 130, 64], 64, 96, 0, 3), ([300, 0, 1, 211], 256, 320, 0, 0),
                                                     ([31, 33, 32], 100, 60, 40, 0), ([1] * 70, 64, 64, 0, 0), ([513], 1408, 264, 0, 130), ([128, 129], 136, 200, 8, 8),
                                                     ([4598], 384, 480, 0, 1), ([3000, 0, 2001], 257, 263, 5, 0), ([2500], 1030, 1001, 0, 0), ([700, 650], 1026, 1032, 1, 1),
                                                     ([900] * 3, 1032, 1035, 0, 0), ([1100], 2048, 2050, 0, 0), ([8000], 129, 130, 0, 0),
                                                     ([4000, 3999], 1032, 136, 1, 0), ([4001], 2056, 4104, 0, 0)])
def test_weight_gradient_of_mx8_rows(lib, counts, m, n, before, extra, dtype):
    rng = np.random.default_rng(m + n)
    G, live, dt = len(counts), sum(counts), DT[dtype]
    rows, a = before + live + extra, before
    ends = before + np.r_[0, np.cumsum(counts)]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    dZ, _ = strided(rows, n, 8, dt)
    dZ[a: a + live].copy_(torch.from_numpy(rng.standard_normal((live, n)) * 0.1).to(dt))
    x = torch.full((max(rows, 1), m), float("nan"), dtype=dt, device="cuda")
    x[a: a + live] = torch.from_numpy(rng.standard_normal((live, m))).to(dt).cuda()
    Q = mx8_of(x) if rows else torch.zeros(256, dtype=torch.uint8, device="cuda")
    xh = mx8_values(*split_mx8(Q, rows, m), m) if rows else np.zeros((0, m))
    zh = host(dZ).numpy()
    desc = px.make_grouped_desc(m, n, G, rows, CODE[dtype], px.GROUPED_X_MX8)
    need = px.poetx_grouped_workspace_bytes(desc)
    dW = torch.full((G, n, m), float("nan"), device="cuda")
    px.poetx_grouped_bwd_weight(desc, Q, dZ, off, dW, False, scratch(need))
    first = dW.clone()
    px.poetx_grouped_bwd_weight(desc, Q, dZ, off, dW, True, scratch(need))
    for g in range(G):
        p, q = ends[g], ends[g + 1]
        ref, mag = zh[p:q].T @ xh[p:q], np.abs(zh[p:q]).T @ np.abs(xh[p:q])
        for got, k in ((first, 1), (dW, 2)):
            err = np.abs(host(got[g]).numpy() - k * ref)
            assert (err <= k * ((q - p + 4) * U24 * mag + 2 * U24 * np.abs(ref)) + 1e-37).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,pad,shift,out_shift", [(136, 3, 0, 0), (136, 8, 1, 0), (136, 8, 0, 1), (131, 5, 3, 0), (131, 5, 0, 2)])
def test_weight_gradient_of_mx8_rows_elsewhere(lib, n, pad, shift, out_shift, dtype):
    """dZ and dW on any alignment, dZ of any leading dimension."""
    rng = np.random.default_rng(n + pad)
    counts, m, dt = [700, 0, 611], 260, DT[dtype]
    rows, ends = sum(counts), np.r_[0, np.cumsum(counts)]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    dZ, _ = strided(rows, n, pad, dt, shift)
    dZ.copy_(torch.from_numpy(rng.standard_normal((rows, n)) * 0.1).to(dt))
    Q = mx8_of(torch.from_numpy(rng.standard_normal((rows, m))).to(dt).cuda())
    xh, zh = mx8_values(*split_mx8(Q, rows, m), m), host(dZ).numpy()
    desc = px.make_grouped_desc(m, n, 3, rows, CODE[dtype], px.GROUPED_X_MX8)
    flat = torch.full((3 * n * m + 8,), 3.0, device="cuda")
    dW = flat[out_shift: out_shift + 3 * n * m].view(3, n, m)
    px.poetx_grouped_bwd_weight(desc, Q, dZ, off, dW, False, scratch(px.poetx_grouped_workspace_bytes(desc)))
    for g in range(3):
        p, q = ends[g], ends[g + 1]
        ref, mag = zh[p:q].T @ xh[p:q], np.abs(zh[p:q]).T @ np.abs(xh[p:q])
        assert (np.abs(host(dW[g]).numpy() - ref) <= (q - p + 4) * U24 * mag + 2 * U24 * np.abs(ref) + 1e-37).all()
    dW.fill_(3.0)
    assert bool((flat == 3.0).all())


# ------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,act", [("bf16", "silu"), ("f32", "gelu")])
def test_training_step(lib, dtype, act):
    """The block as a step uses it: X and G, U kept in eight bits, dX and dW by the grouped products on the stacked weight.  Kept values are exact inputs of what follows."""
    counts, m, n = [70, 0, 33, 129], 96, 160
    b = Block(counts, m, n, dtype, act)
    QG, QU, (G, U) = run_forward_mx8(b)
    QX = mx8_of(b.X)
    xh = torch.from_numpy(mx8_values(*split_mx8(QX, b.rows, m), m))
    GU = torch.empty((b.rows, 2 * n), dtype=b.dt, device="cuda")
    px.poetx_gated_bwd(b.desc(px.GATED_HELD_MX8), b.dH, QG, QU, b.off, GU[:, :n], GU[:, n:])
    zero = torch.zeros_like(G)
    rG, rU, lG, lU = backward_of(act, b.live(b.dH), G, U, zero, zero, b.r / 2)
    near(host(GU), torch.cat([rG, rU], 1), torch.cat([lG, lU], 1), "dG | dU")
    desc = px.make_grouped_desc(m, 2 * n, b.groups, b.rows, CODE[dtype])
    dX = torch.empty((b.rows, m), dtype=b.dt, device="cuda")
    px.poetx_grouped_bwd_input(desc, GU, b.W, b.off, dX, scratch(px.poetx_grouped_workspace_bytes(desc)))
    desc = px.make_grouped_desc(m, 2 * n, b.groups, b.rows, CODE[dtype], px.GROUPED_X_MX8)
    dW = torch.empty((b.groups, 2 * n, m), device="cuda")
    px.poetx_grouped_bwd_weight(desc, QX, GU, b.off, dW, False, scratch(px.poetx_grouped_workspace_bytes(desc)))
    z, ends = host(GU), b.off.tolist()
    for g in range(b.groups):
        p, q = ends[g], ends[g + 1]
        ref, mag = z[p:q] @ b.Wh[g], z[p:q].abs() @ b.Wh[g].abs()
        near(host(dX[p:q]), ref, (2 * n + 2) * U24 * mag + b.r * 1.01 * ref.abs(), "dX")
        ref, mag = z[p:q].t() @ xh[p:q], z[p:q].abs().t() @ xh[p:q].abs()
        near(host(dW[g]), ref, (q - p + 4) * U24 * mag + 2 * U24 * ref.abs(), "dW")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(lib, act):
    """dX, dW of L = <dH, H(X, W)> in fp32 against central differences of the formula in 64 bits along directions v: those are off by t^2 / 6 of a third derivative, with
    t = 1e-4 under 1e-6 of the sizes here, and by 2^-53 / t."""
    counts, m, n = [5, 0, 9], 24, 40
    b = Block(counts, m, n, "f32", act)
    GU = torch.empty((b.rows, 2 * n), device="cuda")
    px.poetx_gated_bwd_recompute(b.desc(), b.dH, b.X, b.W, b.off, GU[:, :n], GU[:, n:], ws=b.ws(b.desc()))
    desc = px.make_grouped_desc(m, 2 * n, b.groups, b.rows, px.F32)
    dX, dW = torch.empty((b.rows, m), device="cuda"), torch.empty((b.groups, 2 * n, m), device="cuda")
    px.poetx_grouped_bwd_input(desc, GU, b.W, b.off, dX)
    px.poetx_grouped_bwd_weight(desc, b.X, GU, b.off, dW, False)
    ends, dH = b.off.tolist(), host(b.dH)

    def loss(x, w):
        total = 0.0
        for g in range(b.groups):
            p, q = ends[g], ends[g + 1]
            gu = x[p:q] @ w[g].t()
            a = activation(act, gu[:, :n], 0.0)[0]
            total += float((dH[p:q] * a * gu[:, n:]).sum())
        return total

    gen, t = torch.Generator().manual_seed(2), 1e-4
    for _ in range(6):
        vx, vw = torch.randn(b.xh.shape, generator=gen, dtype=torch.float64), torch.randn(b.Wh.shape, generator=gen, dtype=torch.float64) / m ** 0.5
        for slope, grad, v in ((lambda s: loss(b.xh + s * vx, b.Wh), host(dX), vx), (lambda s: loss(b.xh, b.Wh + s * vw), host(dW), vw)):
            want = (slope(t) - slope(-t)) / (2 * t)
            size = float((grad.abs() * v.abs()).sum())
            assert abs(want - float((grad * v).sum())) < 4e-6 * size


# ------------------------------------------------------------------------------------ how calls are made
def _calls(b):
    """Every call of the block on one set of tensors, as a function that makes them all, and its outputs."""
    desc, mx8 = b.desc(), b.desc(px.GATED_HELD_MX8)
    ws = torch.empty(max(256, px.poetx_gated_workspace_bytes(desc), px.poetx_gated_workspace_bytes(mx8)), dtype=torch.uint8, device="cuda")
    H = [torch.zeros((b.rows, b.n), dtype=b.dt, device="cuda") for _ in range(4)]
    GU, dGU, dGU8, dGUr = (torch.zeros((b.rows, 2 * b.n), dtype=b.dt, device="cuda") for _ in range(4))
    Q = [torch.zeros(px.poetx_mx8_bytes(b.rows, b.n), dtype=torch.uint8, device="cuda") for _ in range(2)]
    QX = torch.zeros(px.poetx_mx8_bytes(b.rows, b.m), dtype=torch.uint8, device="cuda")
    X = torch.zeros((b.rows, b.m), dtype=b.dt, device="cuda")
    gd = px.make_grouped_desc(b.m, 2 * b.n, b.groups, b.rows, CODE[b.dtype], px.GROUPED_X_MX8)
    gws = torch.empty(max(256, px.poetx_grouped_workspace_bytes(gd)), dtype=torch.uint8, device="cuda")
    dW = torch.zeros((b.groups, 2 * b.n, b.m), device="cuda")
    half = lambda t: t.split(b.n, 1)      # noqa: E731

    def run():
        px.poetx_gated_fwd(desc, b.X, b.W, b.off, H[0], *half(GU), ws=ws)
        px.poetx_gated_bwd(desc, b.dH, *half(GU), b.off, *half(dGU), H[1])
        px.poetx_gated_fwd(mx8, b.X, b.W, b.off, H[2], *Q, ws=ws)
        px.poetx_gated_bwd(mx8, b.dH, *Q, b.off, *half(dGU8), H[3])
        px.poetx_gated_bwd_recompute(desc, b.dH, b.X, b.W, b.off, *half(dGUr), ws=ws)
        px.poetx_mx8_quantize(b.X, QX)
        px.poetx_mx8_dequantize(QX, X)
        if not b.flags:
            px.poetx_grouped_bwd_weight(gd, QX, dGUr, b.off, dW, False, gws)

    return run, [*H, GU, dGU, dGU8, dGUr, *Q, QX, X, dW]


CALLS = [([70, 0, 260], 256, 192, "bf16", "dense"), ([1, 0, 2], 1024, 96, "bf16", "dense"), ([3, 2], 512, 64, "bf16", "mx4"), ([90, 33], 136, 72, "f32", "dense"),
         ([20], 65, 33, "bf16", "dense")]


@pytest.mark.parametrize("counts,m,n,dtype,weight", CALLS)
def test_repeated_on_another_stream_and_in_a_graph(lib, counts, m, n, dtype, weight):
    """The same bits every time: again, on a stream that is not the current one when the tensors are made, and replayed from a graph with eager calls in between."""
    b = Block(counts, m, n, dtype, weight=weight)
    run, outs = _calls(b)
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
    for i in range(4):
        cleared()
        graph.replay()
        same(f"replay {i}")
        run()      # eager work between replays
        same(f"eager {i}")


def test_two_graphs_share_a_workspace(lib):
    """Two captured passes over different inputs with one workspace, replayed in turn on one stream."""
    blocks = [Block([70, 0, 260], 256, 192, "bf16", seed=s) for s in (0, 1)]
    desc = blocks[0].desc(px.GATED_HELD_MX8)
    ws = torch.empty(max(256, px.poetx_gated_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    outs, graphs, want = [], [], []
    for b in blocks:
        H = torch.zeros((b.rows, b.n), dtype=b.dt, device="cuda")
        Q = [torch.zeros(px.poetx_mx8_bytes(b.rows, b.n), dtype=torch.uint8, device="cuda") for _ in range(2)]
        px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, *Q, ws=ws)
        want.append([t.clone() for t in (H, *Q)])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, *Q, ws=ws)
        outs.append((H, *Q))
        graphs.append(g)
    for _ in range(3):
        for i in (0, 1):
            for t in outs[i]:
                t.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(t, w) for t, w in zip(outs[i], want[i]))


def test_rows_past_32_bits(lib):
    """Matrices whose last row starts beyond 2^31 elements."""
    rows, n, m, ld = 1030, 64, 64, 1 << 21
    b = Block([rows], m, n, "bf16")
    wide = [torch.full((rows * ld,), 3.0, dtype=torch.bfloat16, device="cuda").view(rows, ld) for _ in range(2)]
    X, H = wide[0][:, :m], wide[1][:, :n]
    G, U, dG, dU, dH = (wide[1][:, n * i: n * (i + 1)] for i in range(2, 7))
    X.copy_(b.X)
    dH.copy_(b.dH)
    desc = b.desc()
    Hn = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    px.poetx_gated_fwd(desc, X, b.W, b.off, H, ws=b.ws(desc))
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, Hn, ws=b.ws(desc))
    ref, lim = forward_of("silu", b.G, b.U, b.eG, b.eU, b.r / 2)
    near(host(H), ref, lim, "H wide")
    near(host(Hn), ref, lim, "H")
    px.poetx_gated_fwd(desc, X, b.W, b.off, Hn, G, U, ws=b.ws(desc))
    near(host(G), b.G, b.eG + b.r * (b.G.abs() + b.eG), "G kept")
    dGn, dUn = (torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    Gn, Un, dHn = (t.contiguous() for t in (G, U, dH))
    px.poetx_gated_bwd(desc, dHn, Gn, Un, b.off, dG, dU)
    px.poetx_gated_bwd(desc, dH, G, U, b.off, dGn, dUn)
    assert torch.equal(dGn, dG) and torch.equal(dUn, dU)


def test_mx8_past_32_bits(lib):
    """More than 2^31 elements: the last rows come back as the first."""
    rows, cols = 33000, 65600
    x = torch.randn((4, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    X = x.repeat(rows // 4, 1)
    Q = torch.empty(px.poetx_mx8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    px.poetx_mx8_quantize(X, Q)
    X.zero_()
    px.poetx_mx8_dequantize(Q, X)
    want = torch.from_numpy(mx8_values(*oracle_mx8(host(x).numpy()), cols)).to(torch.bfloat16).cuda()
    assert torch.equal(X.view(rows // 4, 4, cols), want.expand(rows // 4, 4, cols))


@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_profiled_and_refused(lib, activation):
    """Stage timing counts the block's launches; a tensor of another shape or type is refused by the binding."""
    b = Block([20, 300], 128, 96, "bf16", activation)
    desc = b.desc()
    H, ws = torch.empty((b.rows, b.n), dtype=b.dt, device="cuda"), b.ws(desc)
    px.poetx_profile_begin(16)
    px.poetx_gated_fwd(desc, b.X, b.W, b.off, H, ws=ws)
    stages = px.poetx_profile_end()
    assert stages["dense"][1] == 1 and stages["dequant"][1] == 0
    with pytest.raises(AssertionError):
        px.poetx_gated_fwd(desc, b.X, b.W, b.off, H.float(), ws=ws)
    with pytest.raises(AssertionError):
        px.poetx_gated_fwd(desc, b.X[:, :64], b.W, b.off, H, ws=ws)
    with pytest.raises(AssertionError):
        px.poetx_gated_fwd(desc, b.X, b.W[:1], b.off, H, ws=ws)
    with pytest.raises(px.PoetxError):
        px.poetx_gated_fwd(desc, b.X, b.W, b.off, b.dH.new_empty(0).set_(b.X.untyped_storage(), 0, (b.rows, b.n), (b.m, 1)), ws=ws)


@pytest.mark.parametrize("held", ["same", "nothing", "mx8"])
def test_gated_experts_example(lib, held):
    """The example layer of gated experts in fp32 against torch autograd in float64.  What is kept in eight bits moves gradients by up to 2^-6 of the largest of 32 elements, and act, act' and
    their products by a few times that: a tenth of the largest gradient bounds it there."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "experts.py")
    spec = importlib.util.spec_from_file_location("experts_example", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    tokens, d, f, E, k = 50, 64, 96, 5, 2
    gen = torch.Generator(device="cuda").manual_seed(4)
    W1, W2 = (torch.stack([ex.merged(torch.randn(s, device="cuda", generator=gen) * 0.1, 16, 3, 0.02, gen) for _ in range(E)]) for s in ((2 * f, d), (d, f)))
    x, dout = (torch.randn((tokens, d), device="cuda", generator=gen) for _ in range(2))
    ids = torch.randint(-1, E, (tokens, k), device="cuda", generator=gen)
    gates = torch.rand((tokens, k), device="cuda", generator=gen)
    layer = ex.GatedExperts(W1, W2, tokens, k, held=held)
    out = layer.forward(x, ids, gates)
    dx, dgate, (dW1, dW2) = layer.backward(dout, weights=True)
    leaves = [t.double().cpu().requires_grad_() for t in (x, gates, W1, W2)]
    xr, gr, W1r, W2r = leaves
    e = ids.cpu().clamp(min=0)
    gu = (W1r[e] * xr[:, None, None, :]).sum(3)
    h = torch.nn.functional.silu(gu[..., :f]) * gu[..., f:]
    ref = ((W2r[e] * h[:, :, None, :]).sum(3) * (gr * (ids.cpu() >= 0)).unsqueeze(2)).sum(1)
    ref.backward(dout.double().cpu())
    for got, want, exact in ((out, ref, True), (dx, xr.grad, held != "mx8"), (dgate, gr.grad, True), (dW1, W1r.grad, held != "mx8"), (dW2, W2r.grad, held != "mx8")):
        assert float((host(got) - want.detach()).abs().max()) <= (1e-5 if exact else 0.1) * float(want.detach().abs().max())
    small = ["--tokens", "70", "--experts", "4", "--d", "256", "--hidden", "192", "--block", "64", "--steps", "1", "--expert", "gated", "--held", held]
    for more in ([], ["--weights", "dense"]):
        assert ex.main(small + more) == 0
