"""The operators of a gated feed-forward block and of activations held in eight bits: both projections with the activation
and the product, their backward pass, the eight-bit form, and the weight gradient that reads it.

Kinds of pass
    fwd       H = act(G) * U with G = X Wg^T, U = X Wu^T, each row of X by its group's pair of weights
    hold      the same in training: G and U are kept for the backward pass, in the type or in eight bits
    bwd       dH and what was kept -> dG, dU and, for the weight gradient of the product that follows, H again
    again     the same where nothing was kept: G and U are made again from X
    mx8       a matrix into 8-bit codes with a power-of-two scale per 32 elements of a row, and back into values
    dweight   dW = [dG dU]^T X of every group, in fp32, where X was kept in eight bits

A case is a dict: kind, rows, m (d_in), n (hidden size), groups, idle (groups, the last ones, that get no rows), dtype
("f32" / "bf16"), act ("silu" / "gelu"), weight ("dense" / "mx4") and held ("same" / "mx8").  `mx8` cases have rows, m and dtype.

The weights of a group lie one below the other, gate then up: groups x 2 n x m.  The plain form pads every group to the
longest and multiplies the batch; a handful of rows gather their weights.
"""
from __future__ import annotations

import math

import torch

own = False


def _ff(name, kind, rows, m, n, groups=1, idle=0, dtype="bf16", act="silu", weight="dense", held="same"):
    return {"name": name, "kind": kind, "rows": rows, "m": m, "n": n, "groups": groups, "idle": idle, "dtype": dtype,
            "act": act, "weight": weight, "held": held}


def listed():
    return [
        # generation, one token through both projections of the 8B-shaped layer: the weights' bytes are all there is
        _ff("gated-token", "fwd", 1, 4096, 14336),
        # generation, one token's eight experts out of 64, weights in four bits
        _ff("gated-experts-token", "fwd", 8, 2048, 1376, groups=64, weight="mx4"),
        # training forward in fp32 of the smallest layer, an odd number of tokens, everything kept
        _ff("gated-f32-hold", "hold", 1999, 512, 1376, dtype="f32", act="gelu", held="same"),
        # training forward over many small experts, an odd number of rows, some experts without any
        _ff("gated-experts-hold", "hold", 8190, 2048, 1376, groups=64, idle=7, held="same"),
        # training forward of a full batch of 4 x 4096 tokens, kept in eight bits: the largest pass
        _ff("gated-batch-hold", "hold", 16384, 4096, 14336, held="mx8"),
        # backward of the smallest layer: a launch and little else
        _ff("bwd-small", "bwd", 1001, 512, 1376, dtype="f32", act="gelu", held="same"),
        # backward of the full batch from what was kept in eight bits
        _ff("bwd-batch", "bwd", 16384, 4096, 14336, held="mx8"),
        # backward where nothing was kept: the 1B-shaped layer
        _ff("bwd-again", "again", 4096, 2048, 5632),
        # one token's hidden state into eight bits and back: two launches and nothing else
        {"name": "mx8-token", "kind": "mx8", "rows": 1, "m": 4096, "dtype": "bf16"},
        # the input of the block for a full batch
        {"name": "mx8-batch", "kind": "mx8", "rows": 16384, "m": 4096, "dtype": "bf16"},
        # weight gradients of experts, their input kept in eight bits
        _ff("dweight-experts", "dweight", 8192, 2048, 1376, groups=16, idle=1, held="mx8"),
        # weight gradients of the 1B-shaped layer, one group, an odd number of rows
        _ff("dweight-layer", "dweight", 4095, 2048, 5632, held="mx8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A feature count: mostly whole 16-byte vectors, at times whatever it is."""
    d = _log(rng, lo, hi)
    return d if rng.random() < 0.15 else max(lo, d // 32 * 32)


def draw(rng):
    kind = rng.choice(("fwd", "fwd", "hold", "hold", "bwd", "bwd", "again", "mx8", "dweight", "dweight"))
    if kind == "mx8":
        m = _size(rng, 32, 14336)
        return {"kind": "mx8", "rows": min(_log(rng, 1, 16384), 16384 * 4096 // m), "m": m, "dtype": rng.choice(("f32", "bf16"))}
    single = rng.random() < 0.2
    m, n = (_size(rng, 64, 2048), _size(rng, 64, 2048)) if single else (_size(rng, 256, 8192), _size(rng, 256, 8192))
    groups = 1 if rng.random() < 0.4 else min(_log(rng, 2, 64), 2 ** 27 // (m * n) + 1)
    rows = min(_log(rng, 1, 4096 if single else 16384), 16384 * 4096 * 4096 // (m * n))
    return {"kind": kind, "rows": rows, "m": m, "n": n, "groups": groups, "idle": rng.randint(0, groups // 4),
            "dtype": "f32" if single else "bf16", "act": rng.choice(("silu", "silu", "gelu")),
            "weight": "mx4" if kind in ("fwd", "hold", "again") and not single and rng.random() < 0.35 else "dense",
            "held": "mx8" if kind == "dweight" or (kind in ("hold", "bwd") and rng.random() < 0.5) else "same"}


# ------------------------------------------------------------------------------------ the formats, plain
# A buffer of four (eight) bits: codes [rows][mp / 2] ([rows][mp]) bytes, mp = m rounded up to 128; from the next
# multiple of 256 bytes on, scale bytes [rows][mp / 32].
#   four bits    value = e2m1(code) * 2^(scale - 127), element 2i in the low half of byte i
#   eight bits   value = code / 64 * 2^(scale - 127), code a signed byte
def _padded(m):
    return -(-m // 128) * 128


def _scale_offset(code_bytes):
    return -(-code_bytes // 256) * 256


def _power(e):
    """2^e in 64 bits, every bit of it, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _blocks(x):
    """rows x m -> the same padded, in blocks of 32, in 64 bits, and floor(log2(largest magnitude)) of each block."""
    x = torch.nn.functional.pad(x.double(), (0, _padded(x.shape[1]) - x.shape[1])).view(x.shape[0], -1, 32)
    top = x.abs().amax(-1)
    return x, top, torch.frexp(top).exponent - 1


def _buffer(codes, scale):
    codes = codes.contiguous().view(-1)
    off = _scale_offset(codes.numel())
    q = torch.zeros(off + scale.numel(), dtype=torch.uint8, device=codes.device)
    q[: codes.numel()] = codes
    q[off:] = scale.to(torch.uint8).view(-1)
    return q


def _parts(q, rows, m, per_byte):
    mp = _padded(m)
    size = rows * mp // per_byte
    return q[:size].view(rows, -1), q[_scale_offset(size):][: rows * mp // 32].view(rows, -1)


def _mx8_codes(x):
    """rows x m -> codes [rows][mp] (signed), scale bytes [rows][mp / 32]."""
    rows = x.shape[0]
    v, top, e = _blocks(x)
    scale = torch.where(top > 0, (e + 127).clamp(0, 254), 0)
    scale = torch.where(top < math.inf, scale, 255)
    code = torch.round(v * _power(133 - scale).unsqueeze(-1)).clamp(-127, 127)      # ties to even
    code = torch.where((scale < 255).unsqueeze(-1), code, 0.0)
    return code.view(rows, -1), scale


def _mx8_values(code, scale, m):
    unit = torch.where(scale < 255, _power(scale.long() - 133), math.nan)
    return (code.view(code.shape[0], -1, 32).double() * unit.unsqueeze(-1)).view(code.shape[0], -1)[:, :m]


def _mx8_pack(x):
    parts = [_mx8_codes(p) for p in x.split(2048)]
    code, scale = (torch.cat(t) for t in zip(*((c.to(torch.int8), s) for c, s in parts)))
    return _buffer(code.view(torch.uint8), scale)


def _mx8_unpack(q, rows, m):
    code, scale = _parts(q, rows, m, 1)
    return _mx8_values(code.view(torch.int8), scale.int(), m).float()


def _mx4_pack(x):
    v, top, e = _blocks(x)
    scale = torch.where(top > 0, (e + 125).clamp(0, 254), 0)
    a = v.abs() * _power(127 - scale).unsqueeze(-1)
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) + 8 * torch.signbit(v)
    code = code.view(x.shape[0], -1)
    return (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8), scale


def _mx4_unpack(q, rows, m):
    b, scale = _parts(q, rows, m, 2)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=q.device)
    code = torch.stack((b & 15, b >> 4), -1).view(rows, -1, 32)
    unit = _power(scale.int() - 127).float()
    return (grid[code.int()] * unit.unsqueeze(-1)).view(rows, -1)[:, :m]


# ------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _tokens(g, rows, m, dtype):
    """Rows of features as a norm leaves them, some features larger than the rest."""
    return _randn(g, (rows, m), torch.exp(0.4 * torch.randn(m, generator=g, device="cuda")), dtype)


def _ids(case, seed):
    """Group of every row: popular and unpopular groups, the last `idle` of them never chosen."""
    g = torch.Generator().manual_seed(seed)
    live = case["groups"] - case["idle"]
    return torch.multinomial(torch.exp(0.5 * torch.randn(live, generator=g)), case["rows"], replacement=True, generator=g)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case, "plan": {}}
    if kind == "mx8":
        s["X"] = _tokens(g, case["rows"], case["m"], _dt(case))
        s["values"] = torch.empty_like(s["X"])
        return s
    rows, m, n, groups, dt = case["rows"], case["m"], case["n"], case["groups"], _dt(case)
    ids = torch.sort(_ids(case, seed)).values
    count = torch.bincount(ids, minlength=groups)
    start = torch.cumsum(count, 0) - count
    s["offsets"] = torch.cat([start, torch.tensor([rows])]).int().cuda()
    s["group"], s["place"], s["longest"] = ids.cuda(), (torch.arange(rows) - start[ids]).cuda(), int(count.max())
    if kind in ("fwd", "hold", "again"):
        s["X"] = _tokens(g, rows, m, dt)
        if case["weight"] == "mx4":
            codes, scale = (torch.cat(t) for t in zip(*(_mx4_pack(_randn(g, (2 * n, m), m ** -0.5, dt)) for _ in range(groups))))
            s["W"] = _buffer(codes, scale)
        else:
            s["W"] = _randn(g, (groups, 2 * n, m), m ** -0.5, dt)
    if kind == "bwd":      # what the forward pass kept
        GU = _randn(g, (rows, 2 * n), 1.0, dt)
        s["G"], s["U"] = (_mx8_pack(GU[:, :n]), _mx8_pack(GU[:, n:])) if case["held"] == "mx8" else (GU[:, :n], GU[:, n:])
    if kind == "hold":
        s["G"], s["U"] = torch.empty((rows, 2 * n), dtype=dt, device="cuda").split(n, 1)
    if kind in ("bwd", "again"):
        s["dH"] = _randn(g, (rows, n), 0.1, dt)
        s["dG"], s["dU"] = torch.empty((rows, 2 * n), dtype=dt, device="cuda").split(n, 1)
    if kind == "dweight":
        s["X"] = _mx8_pack(_tokens(g, rows, m, dt))
        s["dGU"] = _randn(g, (rows, 2 * n), 0.1, dt)
        s["dW"] = torch.empty((groups, 2 * n, m), dtype=torch.float32, device="cuda")
    else:
        s["H"] = torch.empty((rows, n), dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------------------------------ the passes
def _act(case, g):
    """The activation and its derivative: g s(z) with s the logistic function and z = g, or the cubic of the tanh form of gelu."""
    if case["act"] == "silu":
        z, dz = g, 1.0
    else:
        c = 2 * math.sqrt(2 / math.pi)
        z, dz = c * (g + 0.044715 * g * g * g), c * (1 + 3 * 0.044715 * g * g)
    s = 1 / (1 + torch.exp(-z))
    return g * s, s * (1 + g * dz * (1 - s))


def _padded_rows(s, x):
    """[rows][d] -> [groups][longest][d], zeros where a group is shorter."""
    p = torch.zeros((s["case"]["groups"], s["longest"], x.shape[1]), device=x.device)
    p[s["group"], s["place"]] = x
    return p


def _projections(s):
    case = s["case"]
    rows, m, n, groups = case["rows"], case["m"], case["n"], case["groups"]
    x = s["X"].float()
    W = _mx4_unpack(s["W"], groups * 2 * n, m).view(groups, 2 * n, m) if case["weight"] == "mx4" else s["W"]
    if groups == 1:
        gu = x @ W[0].float().t()
    elif rows <= groups:      # a handful of rows: each with its own weight
        gu = (W[s["group"]].float() * x.unsqueeze(1)).sum(2)
    else:
        gu = torch.bmm(_padded_rows(s, x), W.float().transpose(1, 2))[s["group"], s["place"]]
    return gu[:, :n], gu[:, n:]


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "mx8":
        return _mx8_values(*_mx8_codes(s["X"]), case["m"]).to(s["X"].dtype)
    rows, m, n, dt = case["rows"], case["m"], case["n"], _dt(case)
    if kind == "dweight":
        x, dz = _mx8_unpack(s["X"], rows, m), s["dGU"].float()
        if case["groups"] == 1:
            return (dz.t() @ x).unsqueeze(0)
        return torch.bmm(_padded_rows(s, dz).transpose(1, 2).contiguous(), _padded_rows(s, x))
    if kind != "bwd":
        G, U = _projections(s)
    elif case["held"] == "mx8":
        G, U = _mx8_unpack(s["G"], rows, n), _mx8_unpack(s["U"], rows, n)
    else:
        G, U = s["G"].float(), s["U"].float()
    a, da = _act(case, G)
    H = (a * U).to(dt)
    if kind == "fwd":
        return H
    if kind == "hold":
        kept = [_mx8_values(*_mx8_codes(t), n) if case["held"] == "mx8" else t for t in (G, U)]
        return {"H": H, "G": kept[0].to(dt), "U": kept[1].to(dt)}
    dH = s["dH"].float()
    return {"dG": (dH * U * da).to(dt), "dU": (dH * a).to(dt), "H": H}


def _own(s):
    import paper_2603_05500_amd as px
    case, plan = s["case"], s["plan"]
    kind, rows, m = case["kind"], case["rows"], case["m"]

    def scratch(nbytes):
        return torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")

    if kind == "mx8":
        if not plan:
            plan["Q"] = scratch(px.poetx_mx8_bytes(rows, m))
        px.poetx_mx8_quantize(s["X"], plan["Q"])
        px.poetx_mx8_dequantize(plan["Q"], s["values"])
        return s["values"]
    n, groups, dtype = case["n"], case["groups"], px.F32 if case["dtype"] == "f32" else px.BF16
    if kind == "dweight":
        if not plan:
            plan["desc"] = px.make_grouped_desc(m, 2 * n, groups, rows, dtype, px.GROUPED_X_MX8)
            plan["ws"] = scratch(px.poetx_grouped_workspace_bytes(plan["desc"]))
        px.poetx_grouped_bwd_weight(plan["desc"], s["X"], s["dGU"], s["offsets"], s["dW"], False, plan["ws"])
        return s["dW"]
    mx8 = case["held"] == "mx8"
    if not plan:
        flags = (px.GATED_W_MX4 if case["weight"] == "mx4" else 0) | (px.GATED_HELD_MX8 if mx8 else 0)
        plan["desc"] = px.make_gated_desc(m, n, groups, rows, dtype, px.GATED_SILU if case["act"] == "silu" else px.GATED_GELU, flags)
        if kind != "bwd":
            plan["ws"] = scratch(px.poetx_gated_workspace_bytes(plan["desc"]))
        if kind == "hold" and mx8:
            plan["G"], plan["U"] = scratch(px.poetx_mx8_bytes(rows, n)), scratch(px.poetx_mx8_bytes(rows, n))
    if kind == "fwd":
        px.poetx_gated_fwd(plan["desc"], s["X"], s["W"], s["offsets"], s["H"], ws=plan["ws"])
        return s["H"]
    if kind == "hold":
        G, U = (plan["G"], plan["U"]) if mx8 else (s["G"], s["U"])
        px.poetx_gated_fwd(plan["desc"], s["X"], s["W"], s["offsets"], s["H"], G, U, ws=plan["ws"])
        if mx8:
            px.poetx_mx8_dequantize(G, s["G"])
            px.poetx_mx8_dequantize(U, s["U"])
        return {"H": s["H"], "G": s["G"], "U": s["U"]}
    if kind == "bwd":
        px.poetx_gated_bwd(plan["desc"], s["dH"], s["G"], s["U"], s["offsets"], s["dG"], s["dU"], s["H"])
    else:
        px.poetx_gated_bwd_recompute(plan["desc"], s["dH"], s["X"], s["W"], s["offsets"], s["dG"], s["dU"], s["H"], ws=plan["ws"])
    return {"dG": s["dG"], "dU": s["dU"], "H": s["H"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind, rows, m = case["kind"], case["rows"], case["m"]
    es = 4 if case["dtype"] == "f32" else 2
    if kind == "mx8":
        return {"bytes": 2 * rows * m * es, "flops": 0}
    n, eight = case["n"], 33 / 32
    live = min(rows, case["groups"] - case["idle"])
    held = eight if case["held"] == "mx8" else es
    if kind == "bwd":
        return {"bytes": rows * n * (es + 2 * held + 3 * es), "flops": 0}
    product = 2 * rows * m * 2 * n
    if kind == "dweight":
        return {"bytes": rows * (m * eight + 2 * n * es) + case["groups"] * 2 * n * m * 4, "flops": product}
    weights = live * 2 * n * m * (17 / 32 if case["weight"] == "mx4" else es)
    out = {"fwd": 1, "hold": 3, "again": 4}[kind]      # `again` reads dH and writes three
    return {"bytes": rows * m * es + weights + rows * n * es * out, "flops": product}


# ------------------------------------------------------------------------------------ in 64 bits, from the definitions
def _exact_scales(q, rows, m, size):
    e = q[-(-size // 256) * 256:][: rows * (-(-m // 128) * 4)].view(rows, -1).long() - 127
    return torch.repeat_interleave(torch.bitwise_left_shift(e + 1023, 52).view(torch.float64), 32, 1)


def _exact_read8(q, rows, m):
    mp = -(-m // 128) * 128
    byte = q[: rows * mp].view(rows, mp).double()
    return ((byte - 256 * (byte > 127)) / 64 * _exact_scales(q, rows, m, rows * mp))[:, :m]


def _exact_read4(q, rows, m):
    mp = -(-m // 128) * 128
    byte = q[: rows * mp // 2].view(rows, mp // 2, 1).int()
    code = torch.cat([byte % 16, byte // 16], 2).view(rows, mp)
    sign, exp, man = code // 8, code // 2 % 4, code % 2
    mag = torch.where(exp == 0, 0.5 * man, (1 + 0.5 * man) * torch.exp2(exp.double() - 1))
    return ((1 - 2 * sign) * mag * _exact_scales(q, rows, m, rows * mp // 2))[:, :m]


def _exact_held(v):
    """Values of 64 bits -> the nearest multiples of 2^(e - 6), at most 127 of them, with 2^e <= the largest of 32 < 2^(e + 1)."""
    rows, m = v.shape
    out = torch.empty_like(v)
    for j in range(0, m, 32):
        b = v[:, j: j + 32]
        top = b.abs().max(1, keepdim=True).values
        unit = torch.where(top > 0, top / torch.frexp(top).mantissa / 128, 1.0)      # the mantissa lies in [1/2, 1)
        k = b / unit
        low = torch.floor(k)
        k = torch.where((k - low > 0.5) | ((k - low == 0.5) & (low % 2 != 0)), low + 1, low)
        out[:, j: j + 32] = torch.where(top > 0, torch.minimum(torch.maximum(k, torch.full_like(k, -127)), torch.full_like(k, 127)) * unit, 0.0)
    return out


def exact(case, seed):
    kind, rows, m = case["kind"], case["rows"], case["m"]
    s = prepare(case, seed)
    if kind == "mx8":
        return _exact_held(s["X"].double())
    n, groups, ends = case["n"], case["groups"], s["offsets"].tolist()
    spans = [(g, ends[g], ends[g + 1]) for g in range(groups) if ends[g + 1] > ends[g]]
    if kind == "dweight":
        x, dz = _exact_read8(s["X"], rows, m), s["dGU"].double()
        dW = torch.zeros((groups, 2 * n, m), dtype=torch.float64, device="cuda")
        for g, a, b in spans:
            dW[g] = dz[a:b].t() @ x[a:b]
        return dW
    if kind == "bwd":
        G, U = (_exact_read8(t, rows, n) if case["held"] == "mx8" else t.double() for t in (s["G"], s["U"]))
    else:
        x = s["X"].double()
        G, U = (torch.empty((rows, n), dtype=torch.float64, device="cuda") for _ in range(2))
        for g, a, b in spans:
            if case["weight"] == "mx4":      # this group's rows of the buffer, as a buffer of their own
                half, sc = (-(-m // 128) * 128) // 2, -(-m // 128) * 4
                off = -(-groups * 2 * n * half // 256) * 256
                W = _exact_read4(torch.cat([s["W"][g * 2 * n * half: (g + 1) * 2 * n * half], torch.zeros(-2 * n * half % 256, dtype=torch.uint8, device="cuda"),
                                            s["W"][off + g * 2 * n * sc: off + (g + 1) * 2 * n * sc]]), 2 * n, m)
            else:
                W = s["W"][g].double()
            G[a:b], U[a:b] = x[a:b] @ W[:n].t(), x[a:b] @ W[n:].t()
    if case["act"] == "silu":
        share = torch.sigmoid(G)
        slope = share * (1 + G * torch.sigmoid(-G))
        a = G * share
    else:
        root = math.sqrt(2 / math.pi)
        t = torch.tanh(root * (G + 0.044715 * G ** 3))
        a = 0.5 * G * (1 + t)
        slope = 0.5 * (1 + t) + 0.5 * G * (1 - t * t) * root * (1 + 3 * 0.044715 * G ** 2)
    H = a * U
    if kind == "fwd":
        return H
    if kind == "hold":
        kept = (_exact_held(G), _exact_held(U)) if case["held"] == "mx8" else (G, U)
        return {"H": H, "G": kept[0], "U": kept[1]}
    dH = s["dH"].double()
    return {"dG": dH * U * slope, "dU": dH * a, "H": H}
