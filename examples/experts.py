"""A layer of experts on POET-X weights, forward and backward: the products that a training step makes of it.

    python examples/experts.py                      # experts in four bits, activations in bf16
    python examples/experts.py --activations mx4    # activations of the forward products in four bits as well
    python examples/experts.py --weights dense      # experts that are trained themselves: weight gradients too

Each expert is y = W2 relu(W1 x)^2.  Its base weights carry orthogonal factors (blocks of a Cayley-Neumann series under a
permutation; random here), which are folded in once, as in the outer loop's merge step, and not trained any further; frozen
experts are then kept in four bits, and gradients go to the inputs and the router's shares.  A router gives every token its experts; tokens are put in the experts' order on the device, and the products of all
experts are one launch each, whatever the router says: no group size ever comes to the host.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_05500_amd as px  # noqa: E402


def _scratch(nbytes):
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")


def merged(W, block, k, sigma, gen):
    """W (n x m) with random orthogonal factors of `block`-sided blocks folded into both sides."""
    n, m = W.shape
    side, code = {}, px.dtype_code(W)
    precision = px.CNP_FP32 if code == px.F32 else px.CNP_BF16
    for name, d in (("R", m), ("P", n)):
        nb = -(-d // block)
        theta = torch.randn((nb, block * (block - 1) // 2), device="cuda", generator=gen) * sigma
        blocks = torch.empty((nb, block, block) if code == px.F32 else (nb, 2, block, block), dtype=W.dtype, device="cuda")
        px.poetx_cnp_build(theta, d, block, k, precision, *((blocks, None) if code == px.F32 else (None, blocks)),
                           ws=_scratch(px.poetx_cnp_workspace_bytes(d, block)))
        side[name] = torch.randperm(d, device="cuda", generator=gen).int(), blocks
    out = torch.empty_like(W)
    px.poetx_merge_weight(W, out, side["R"][0], side["P"][0], side["R"][1], side["P"][1], block,
                          _scratch(px.poetx_merge_workspace_bytes(n, m, code)))
    return out


class Grouped:
    """Z_r = W_g X_r over the rows of every group g; W: groups x d_out x d_in, kept in four bits if asked."""

    def __init__(self, W, rows, mx4=False, x_mx4=False):
        groups, n, m = W.shape
        flags = (px.GROUPED_W_MX4 if mx4 else 0) | (px.GROUPED_X_MX4 if x_mx4 else 0)
        self.desc = px.make_grouped_desc(m, n, groups, rows, px.dtype_code(W), flags)
        self.ws = _scratch(px.poetx_grouped_workspace_bytes(self.desc))
        self.dtype, self.W = W.dtype, W
        if mx4:
            self.W = torch.empty(px.poetx_mx4_bytes(groups * n, m), dtype=torch.uint8, device="cuda")
            px.poetx_mx4_quantize(W.view(groups * n, m), self.W)

    def _rows(self, d):
        return torch.zeros((self.desc.rows, d), dtype=self.dtype, device="cuda")      # rows of no expert stay zero

    def forward(self, X, offsets):
        Z = self._rows(self.desc.d_out)
        px.poetx_grouped_fwd(self.desc, X, self.W, offsets, Z, self.ws)
        return Z

    def input_gradient(self, dZ, offsets):
        dX = self._rows(self.desc.d_in)
        px.poetx_grouped_bwd_input(self.desc, dZ, self.W, offsets, dX, self.ws)
        return dX

    def weight_gradient(self, X, dZ, offsets):
        dW = torch.empty(self.W.shape, device="cuda")
        px.poetx_grouped_bwd_weight(self.desc, X, dZ, offsets, dW, False, self.ws)
        return dW


class Experts:
    def __init__(self, W1, W2, tokens, top_k, mx4=False, x_mx4=False):
        self.groups, self.top_k, rows = W1.shape[0], top_k, tokens * top_k
        self.up, self.down = Grouped(W1, rows, mx4, x_mx4), Grouped(W2, rows, mx4, x_mx4)
        self.offsets = torch.empty(self.groups + 1, dtype=torch.int32, device="cuda")
        self.order = torch.empty(rows, dtype=torch.int32, device="cuda")
        self.order_ws = _scratch(px.poetx_group_order_workspace_bytes(rows, self.groups))

    def forward(self, x, ids, gates):
        """x: tokens x d; ids, gates: tokens x top_k, the experts of a token (-1: none) and their shares."""
        px.poetx_group_order(ids.reshape(-1).int(), self.offsets, self.order, self.order_ws)
        at = self.order.long()
        self.live = (at >= 0).unsqueeze(1)                       # rows past the last expert's
        self.choice = at.clamp(min=0)
        self.token = self.choice // self.top_k
        self.gate = gates.reshape(-1)[self.choice].unsqueeze(1) * self.live
        self.x = x[self.token]
        self.h = self.up.forward(self.x, self.offsets)
        self.a = self.h.clamp(min=0) ** 2
        self.y = self.down.forward(self.a, self.offsets)
        return torch.zeros_like(x, dtype=torch.float32).index_add_(0, self.token, self.y.float() * self.gate)

    def backward(self, dout, weights=False):
        """dout: tokens x d fp32 -> gradients of x, of the gates and, if asked, of both weights."""
        d = dout[self.token]
        dgate = torch.zeros(len(self.choice), device="cuda").index_add_(0, self.choice, ((d * self.y.float()).sum(1, keepdim=True) * self.live).squeeze(1))
        dy = (d * self.gate).to(self.y.dtype)
        dh = self.down.input_gradient(dy, self.offsets) * (2 * self.h.clamp(min=0))
        dx = torch.zeros_like(dout).index_add_(0, self.token, self.up.input_gradient(dh, self.offsets).float() * self.live)
        dW = (self.up.weight_gradient(self.x, dh, self.offsets), self.down.weight_gradient(self.a, dy, self.offsets)) if weights else None
        return dx, dgate.view(-1, self.top_k), dW


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top-k", type=int, default=2)
    ap.add_argument("--d", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=1408)
    ap.add_argument("--block", type=int, default=128)
    ap.add_argument("--weights", choices=("mx4", "dense"), default="mx4")
    ap.add_argument("--activations", choices=("same", "mx4"), default="same")
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args(argv)
    if a.activations == "mx4" and a.weights != "mx4":
        ap.error("activations in four bits need weights in four bits")
    gen = torch.Generator(device="cuda").manual_seed(0)
    W1, W2 = (torch.stack([merged((torch.randn(s, device="cuda", generator=gen) * 0.02).bfloat16(), a.block, 4, 0.01, gen) for _ in range(a.experts)])
              for s in ((a.hidden, a.d), (a.d, a.hidden)))
    layer = Experts(W1, W2, a.tokens, a.top_k, a.weights == "mx4", a.activations == "mx4")
    router = torch.randn((a.d, a.experts), device="cuda", generator=gen) / a.d ** 0.5
    x = torch.randn((a.tokens, a.d), device="cuda", generator=gen).bfloat16()
    target = torch.randn((a.tokens, a.d), device="cuda", generator=gen) * 0.05

    def step():
        gates, ids = torch.topk(torch.softmax(x.float() @ router, 1), a.top_k, dim=1)
        out = layer.forward(x, ids, gates)
        dout = (out - target) / out.numel()
        return out, layer.backward(dout, weights=a.weights == "dense")

    out, grads = step()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        out, grads = step()
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) / a.steps * 1e3
    finite = all(bool(torch.isfinite(v).all()) for v in (out, grads[0], grads[1], *(grads[2] or ())))
    print(f"{a.tokens} tokens, {a.top_k} of {a.experts} experts of {a.hidden} x {a.d}, weights {a.weights}, activations {a.activations}: "
          f"loss {float(((out - target) ** 2).mean()):.5f}, {ms:.2f} ms per forward and backward, {'finite' if finite else 'NOT FINITE'}")
    return 0 if finite else 1


if __name__ == "__main__":
    sys.exit(main())
