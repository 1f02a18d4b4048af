"""A layer of experts built from the library's routed expert products.

    y[t] = sum over the experts e of token t of R[t, e] * (silu(x[t] W1_e^T) W2_e^T)

R is the routing matrix. The layer is trained on a synthetic target (plain
gradient descent, gradients from the library's kernels), then served token by
token in 16 bits and in 8 bits, and the routing matrix is multiplied with its
transpose to count the experts used together.

Usage: python examples/expert_layer.py [--tokens T] [--experts E] [--top-k K]
[--hidden D] [--inner F] [--steps S]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_22866_amd import gmagnus as g  # noqa: E402


class ExpertLayer:
    """Weights in bfloat16 (w1: experts x inner x hidden, w2: experts x hidden x inner), the router in float32."""

    def __init__(self, hidden: int, inner: int, experts: int, top_k: int, gen: torch.Generator):
        def rand(*shape, scale):
            return torch.randn(shape, device="cuda", generator=gen) * scale

        self.top_k = top_k
        self.router = rand(hidden, experts, scale=hidden ** -0.5)
        self.w1 = rand(experts, inner, hidden, scale=hidden ** -0.5).bfloat16()
        self.w2 = rand(experts, hidden, inner, scale=inner ** -0.5).bfloat16()

    def forward(self, x: torch.Tensor):
        """The layer's result and what backward() needs."""
        logits = x.float() @ self.router
        r = g.route(logits, self.top_k)
        h = g.group_product(x, self.w1, r.group_ptr, index=r.token)
        a = torch.nn.functional.silu(h)
        y = g.group_product(a, self.w2, r.group_ptr)
        return g.combine(y, r.row_ptr, r.slot, r.weight), (x, logits, r, h, a, y)

    def backward(self, d_out: torch.Tensor, saved):
        """Gradients of (x, router, w1, w2)."""
        x, logits, r, h, a, y = saved
        d_y, d_weight = g.combine_backward(y, r.row_ptr, r.slot, r.weight, d_out)
        d_a = g.group_product(d_y, self.w2, r.group_ptr, transposed=True)
        d_w2 = g.group_outer(d_y, a, r.group_ptr, out_dtype=torch.float32)
        s = torch.sigmoid(h.float())
        d_h = (d_a.float() * s * (1 + h.float() * (1 - s))).bfloat16()
        d_w1 = g.group_outer(d_h, x, r.group_ptr, index=r.token, out_dtype=torch.float32)
        d_rows = g.group_product(d_h, self.w1, r.group_ptr, transposed=True)
        d_logits = g.route_backward(logits, r, d_weight)
        d_x = g.combine(d_rows, r.row_ptr, r.slot).float() + d_logits @ self.router.t()
        return d_x, x.float().t() @ d_logits, d_w1, d_w2

    def quantised(self):
        """The layer's weights as E4M3 with a scale for each block of 128 x 128, made once for serving."""
        return g.quantise_blocks(self.w1, 128), g.quantise_blocks(self.w2, 128)

    def serve(self, x: torch.Tensor, weights=None):
        """forward() without what training keeps; in 8 bits with the weights of quantised()."""
        if weights is None:
            return self.forward(x)[0]
        (q1, s1), (q2, s2) = weights
        r = g.route(x.float() @ self.router, self.top_k)
        xq, xs = g.quantise_blocks(x)
        a = torch.nn.functional.silu(g.group_product_fp8(xq, xs, q1, s1, r.group_ptr, index=r.token))
        aq, as_ = g.quantise_blocks(a)
        return g.combine(g.group_product_fp8(aq, as_, q2, s2, r.group_ptr), r.row_ptr, r.slot, r.weight)


def used_together(r: g.Routing) -> torch.Tensor:
    """How many tokens use experts i and j together: R^T R with weights 1, by the library's sparse product."""
    R, Rt = r.matrix(), r.transposed()
    R.val, Rt.val = torch.ones_like(R.val), torch.ones_like(Rt.val)
    row_ptr, col, val = g.spgemm(Rt, R)
    out = torch.zeros(r.n_experts, r.n_experts, device="cuda")
    rows = torch.repeat_interleave(torch.arange(r.n_experts, device="cuda"), row_ptr[1:] - row_ptr[:-1])
    out[rows, col.long()] = val
    return out


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top-k", type=int, default=2)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--inner", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--rate", type=float, default=0.5)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = ExpertLayer(a.hidden, a.inner, a.experts, a.top_k, gen)
    x = torch.randn(a.tokens, a.hidden, device="cuda", generator=gen).bfloat16()
    target = torch.tanh(x.float() @ torch.randn(a.hidden, a.hidden, device="cuda", generator=gen) * a.hidden ** -0.5)
    w1, w2 = layer.w1.float(), layer.w2.float()
    losses = []
    for step in range(a.steps):
        out, saved = layer.forward(x)
        diff = out.float() - target
        losses.append(float(diff.square().mean()))
        _, d_router, d_w1, d_w2 = layer.backward((diff * (2.0 / a.hidden)).bfloat16(), saved)
        scale = a.rate * a.experts / a.tokens
        layer.router -= scale * d_router
        w1 -= scale * d_w1
        w2 -= scale * d_w2
        layer.w1, layer.w2 = w1.bfloat16(), w2.bfloat16()
        if step % 10 == 0 or step == a.steps - 1:
            print("step %d  loss %.4f" % (step, losses[-1]), flush=True)
    whole = layer.serve(x[:8])
    one = torch.cat([layer.serve(x[i:i + 1]) for i in range(8)])
    eight = layer.serve(x[:8], layer.quantised())
    off = float((one.float() - whole.float()).norm() / whole.float().norm())
    off8 = float((eight.float() - whole.float()).norm() / whole.float().norm())
    together = used_together(g.route(x.float() @ layer.router, a.top_k))
    print("one token at a time: %.1e off the batch; in 8 bits: %.1e off" % (off, off8))
    print("busiest expert: %d tokens; most used pair: %d tokens" % (
        int(together.diagonal().max()), int((together - together.diagonal().diag()).max())))
    return {"losses": losses, "one": off, "eight": off8, "together": together}


if __name__ == "__main__":
    main()
