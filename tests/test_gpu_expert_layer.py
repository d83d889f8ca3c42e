"""The example block: its gradients against torch's in 64 bits, and training with it."""
import os
import sys

import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import expert_layer
    finally:
        sys.path.pop(0)
    return expert_layer


def test_block_against_autograd():
    """fp32: output, and the change of the loss along the update that a step made"""
    ex = example()
    device()
    block = ex.Block(48, 40, 6, 2, torch.float32, seed=1)
    names = ["up", "up_bias", "down", "gate_up", "out", "router"]
    x = torch.randn((70, 48), generator=torch.Generator().manual_seed(5)).cuda()
    ids = block.route(x)[0].cpu()
    p = {n: lu.d(getattr(block, n)).clone().requires_grad_(True) for n in names}
    x64 = lu.d(x).requires_grad_(True)
    shared = lu.act(x64 @ p["up"].t() + p["up_bias"], "gelu") @ p["down"].t() + x64
    wt = torch.softmax((x64 @ p["router"].t()).gather(1, ids), 1)
    rows = []
    for t in range(70):
        r = shared[t]
        for j in range(2):
            e = int(ids[t, j])
            z = p["gate_up"][e] @ x64[t]
            r = r + wt[t, j] * (p["out"][e] @ (lu.act(z[:40], "silu") * z[40:]))
        rows.append(r)
    y = torch.stack(rows)
    target = torch.zeros_like(y)
    loss = ((y - target) ** 2).mean()
    loss.backward()
    got = block.serve(x)
    assert float((lu.d(got) - y.detach()).abs().max()) < 1e-4
    before = {n: lu.d(getattr(block, n)).clone() for n in names}
    assert abs(block.step(x, target.float().cuda(), rate=1.0) - loss.item()) < 1e-5 * loss.item()
    for n in names:
        step = before[n] - lu.d(getattr(block, n))
        # an update of 1 in 1e6 of a weight keeps 2^-24 of the weight
        tol = 2e-5 * float(p[n].grad.abs().max()) + 2.0 ** -23 * float(before[n].abs().max())
        assert float((step - p[n].grad).abs().max()) < tol, n
    assert float((lu.d(block.dx) - x64.grad).abs().max()) < 2e-5 * float(x64.grad.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_training_reduces_the_loss(dtype):
    losses = example().main(["--tokens", "512", "--width", "256", "--hidden", "320", "--experts", "8",
                             "--steps", "6", "--dtype", dtype])
    assert all(b < a for a, b in zip(losses, losses[1:]))
