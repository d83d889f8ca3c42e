"""A small language model of a layer of experts, trained and served on the library's operators.

    x = embedding[token];  h = x + experts(norm(x));  loss = -log softmax(W norm(h))[next token]

The experts are chosen by sigmoid scores (``expert_route``) with a bias that is moved
towards even use; the rest of their layer is ``expert_sort``, ``expert_gather``,
``grouped_linear`` and ``expert_combine``; the norms are ``layer_norm``, and the loss is
``linear_cross_entropy``, which never stores the logits.  ``gradients`` writes the backward pass
out; ``serve`` gives the next token's logits for a few tokens.

    python examples/language_model.py                 # bf16, 4096 tokens, 32768 words
    python examples/language_model.py --tokens 512 --width 256 --vocab 1000
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_06510_amd as oz  # noqa: E402


class Model:
    PARAMETERS = ("embedding", "norm1", "norm1_bias", "router", "gate_up", "down", "norm2",
                  "norm2_bias", "out")

    def __init__(self, vocab, width, hidden, experts, top_k, dtype, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape, scale=None):
            w = torch.randn(shape, generator=gen, device="cuda")
            return (w * (shape[-1] ** -0.5 if scale is None else scale)).to(dtype)
        self.experts, self.top_k = experts, top_k
        self.embedding = weight(vocab, width, scale=1.0)
        self.norm1, self.norm1_bias = torch.ones_like(self.embedding[0]), weight(width, scale=0.1)
        self.router = weight(experts, width)
        self.gate_up, self.down = weight(experts, 2 * hidden, width), weight(experts, width, hidden)
        self.norm2, self.norm2_bias = torch.ones_like(self.norm1), weight(width, scale=0.1)
        self.out = weight(vocab, width)
        self.balance = torch.zeros(experts, device="cuda")   # not a parameter: no gradient

    def hidden(self, tokens):
        """Everything up to the norm before the loss, and what the gradients need of it."""
        s = {"x": self.embedding[tokens]}
        s["n"], s["stats1"] = oz.layer_norm(s["x"], self.norm1, self.norm1_bias, save_stats=True)
        s["logits"] = oz.linear(s["n"], self.router)
        s["ids"], s["weights"] = oz.expert_route(s["logits"], self.top_k, bias=self.balance,
                                                 score="sigmoid")
        s["order"] = order = oz.expert_sort(s["ids"], self.experts)
        s["xs"] = oz.expert_gather(s["n"], order)
        s["g"], s["z"] = oz.grouped_linear(s["xs"], self.gate_up, order.offsets, activation="silu",
                                           gated=True, save_preactivation=True)
        s["ys"] = oz.grouped_linear(s["g"], self.down, order.offsets)
        s["h"] = oz.expert_combine(s["ys"], order, s["weights"], residual=s["x"])
        s["f"], s["stats2"] = oz.layer_norm(s["h"], self.norm2, self.norm2_bias, save_stats=True)
        return s

    def serve(self, tokens):
        """The next word's logits."""
        return oz.linear(self.hidden(tokens)["f"], self.out)

    def loss(self, tokens, targets):
        """Each token's loss; 0 where the target is negative."""
        return oz.linear_cross_entropy(self.hidden(tokens)["f"], self.out, targets)[0]

    def gradients(self, tokens, targets):
        """(mean loss of the tokens that count, gradients by name, order of the experts)"""
        s = self.hidden(tokens)
        order, off = s["order"], s["order"].offsets
        loss, lse = oz.linear_cross_entropy(s["f"], self.out, targets)
        count = (targets >= 0).sum().clamp(min=1)
        dloss = ((targets >= 0) / count).float()
        d = {}
        df, d["out"] = oz.linear_cross_entropy_backward(dloss, s["f"], self.out, targets, lse)
        dh, d["norm2"], d["norm2_bias"] = oz.layer_norm_backward(df, s["h"], s["stats2"],
                                                                 weight=self.norm2)
        dys, dweights = oz.expert_combine_backward(dh, s["ys"], order, s["weights"])
        dg, d["down"], _ = oz.grouped_linear_backward(dys, s["g"], self.down, off, need_dbias=False)
        dxs, d["gate_up"], _ = oz.grouped_linear_backward(dg, s["xs"], self.gate_up, off,
                                                          preactivation=s["z"], activation="silu",
                                                          gated=True, need_dbias=False)
        dlogits = oz.expert_route_backward(dweights, s["logits"], s["ids"], score="sigmoid")
        dr, d["router"], _ = oz.linear_backward(dlogits, s["n"], self.router, need_dbias=False)
        dn = oz.expert_combine(dxs, order, residual=dr)   # the gather's gradient, and the router's
        dx, d["norm1"], d["norm1_bias"] = oz.layer_norm_backward(dn, s["x"], s["stats1"],
                                                                 weight=self.norm1, residual=dh)
        d["embedding"] = torch.zeros_like(self.embedding).index_add_(0, tokens, dx)
        return loss.sum() / count, d, order

    def step(self, tokens, targets, rate, balance_rate=0.01):
        """One step of gradient descent; returns the mean loss."""
        loss, d, order = self.gradients(tokens, targets)
        for name in self.PARAMETERS:
            getattr(self, name).sub_(d[name] * rate)
        load = (order.offsets[1:] - order.offsets[:-1]).float()
        self.balance += balance_rate * torch.sign(load.mean() - load)
        return float(loss)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32768)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top-k", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--rate", type=float, default=0.5)
    ap.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    a = ap.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[a.dtype]
    model = Model(a.vocab, a.width, a.hidden, a.experts, a.top_k, dtype, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    text = torch.randint(0, a.vocab, (a.tokens + 1,), generator=gen, device="cuda")
    tokens, targets = text[:-1].clone(), text[1:].clone()
    losses = [model.step(tokens, targets, a.rate) for _ in range(a.steps)]
    print("loss", " ".join(f"{v:.4f}" for v in losses))
    print("next token", int(model.serve(tokens[-1:])[0].float().argmax()))
    return losses


if __name__ == "__main__":
    main()
