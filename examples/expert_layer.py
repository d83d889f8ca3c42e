"""A feed-forward block with experts, trained and served on the library's operators.

    y = x + shared(x) + sum over the chosen experts of weight * expert(x)

The shared layer is a dense gelu layer (``linear``); the experts are gated silu
layers (``expert_sort``, ``expert_gather``, ``grouped_linear``, ``expert_combine``).
``step`` runs one block forward and backward with the gradients written out and a
plain gradient-descent update; ``serve`` is the same block for a few tokens.

    python examples/expert_layer.py                 # bf16, 4096 tokens
    python examples/expert_layer.py --tokens 512 --width 256 --experts 8
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_06510_amd as oz  # noqa: E402


class Block:
    def __init__(self, width, hidden, experts, top_k, dtype, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).to(dtype)
        self.experts, self.top_k = experts, top_k
        self.router = weight(experts, width)
        self.up, self.up_bias = weight(hidden, width), torch.zeros(hidden, dtype=dtype, device="cuda")
        self.down = weight(width, hidden)
        self.gate_up = weight(experts, 2 * hidden, width)   # gates, then values
        self.out = weight(experts, width, hidden)

    def route(self, x):
        """The experts of every token, their weights, and the order by expert."""
        top, ids = torch.topk(oz.linear(x, self.router).float(), self.top_k, dim=1)
        return ids, torch.softmax(top, dim=1), oz.expert_sort(ids, self.experts)

    def serve(self, x):
        _, weights, order = self.route(x)
        shared = oz.linear(oz.linear(x, self.up, bias=self.up_bias, activation="gelu"), self.down,
                           residual=x)
        h = oz.grouped_linear(oz.expert_gather(x, order), self.gate_up, order.offsets,
                              activation="silu", gated=True)
        ys = oz.grouped_linear(h, self.out, order.offsets)
        return oz.expert_combine(ys, order, weights, residual=shared, out=shared)

    def step(self, x, target, rate):
        """One step of gradient descent on mean((y - target)^2); returns the loss."""
        ids, weights, order = self.route(x)
        off = order.offsets
        h, hz = oz.linear(x, self.up, bias=self.up_bias, activation="gelu", save_preactivation=True)
        shared = oz.linear(h, self.down, residual=x)
        xs = oz.expert_gather(x, order)
        g, gz = oz.grouped_linear(xs, self.gate_up, off, activation="silu", gated=True,
                                  save_preactivation=True)
        ys = oz.grouped_linear(g, self.out, off)
        y = oz.expert_combine(ys, order, weights, residual=shared)

        err = y.float() - target.float()
        dy = (err * (2.0 / err.numel())).to(y.dtype)
        dys, dweights = oz.expert_combine_backward(dy, ys, order, weights)
        dg, d_out, _ = oz.grouped_linear_backward(dys, g, self.out, off, need_dbias=False)
        dxs, d_gate_up, _ = oz.grouped_linear_backward(dg, xs, self.gate_up, off, preactivation=gz,
                                                       activation="silu", gated=True,
                                                       need_dbias=False)
        dh, d_down, _ = oz.linear_backward(dy, h, self.down, need_dbias=False)
        dx, d_up, d_bias = oz.linear_backward(dh, x, self.up, preactivation=hz, activation="gelu")
        # the block's input gradient, for the layer before: the residual's, the shared
        # layer's, the experts' (the gather's gradient is a combine), the router's
        dscores = weights * (dweights - (dweights * weights).sum(1, keepdim=True))
        dlogits = torch.zeros((x.shape[0], self.experts), device="cuda")
        dlogits.scatter_(1, ids, dscores)
        dr, d_router, _ = oz.linear_backward(dlogits.to(x.dtype), x, self.router, need_dbias=False)
        self.dx = oz.expert_combine(dxs, order, residual=dy + dx + dr)

        for w, d in ((self.up, d_up), (self.up_bias, d_bias), (self.down, d_down),
                     (self.gate_up, d_gate_up), (self.out, d_out), (self.router, d_router)):
            w -= rate * d
        return float((err * err).mean())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top-k", type=int, default=2)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--rate", type=float, default=4.0)
    ap.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    a = ap.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[a.dtype]
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.tokens, a.width), generator=gen, device="cuda").to(dtype)
    teacher = Block(a.width, a.hidden, a.experts, a.top_k, dtype, seed=2)
    student = Block(a.width, a.hidden, a.experts, a.top_k, dtype, seed=3)
    target = teacher.serve(x)
    losses = [student.step(x, target, a.rate) for _ in range(a.steps)]
    print("loss", " ".join(f"{v:.4f}" for v in losses))
    print("one token", tuple(student.serve(x[:1]).shape))
    return losses


if __name__ == "__main__":
    main()
