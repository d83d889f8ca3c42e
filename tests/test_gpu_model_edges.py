"""The model operators at the ends of their range."""
import pytest
import torch

from tests.gpu_util import device
from tests.test_gpu_router import check_route

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------- router

@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(4, 2), (8, 4), (64, 32), (96, 8), (256, 8), (1024, 4)])
def test_group_sums_beyond_32_bits(E, groups, score):
    """Finite biases whose sums of two are not finite in 32 bits: groups compare as in 64."""
    per, g = E // groups, torch.Generator().manual_seed(E)
    l = torch.randn((5, E), generator=g).to(device())
    for sign in (1.0, -1.0):
        # the groups' sums ascend, from below 3.4e38 to beyond: 2 x 1.6e38 to 2 x 3.2e38
        size = 1.6e38 + 1.6e38 * torch.arange(groups) / max(groups - 1, 1)
        bias = (sign * size).float().repeat_interleave(per).to(device())
        for top in {1, groups // 2}:
            check_route(l, bias, min(2, per), score, groups, top, 2)
        # one expert of each group apart, the rest out of the way: sums of unlike two
        bias[::per] *= 1.01
        check_route(l, bias, 2, score, groups, 1, 2)
        # all beyond, and only some of them different
        bias = torch.full((E,), sign * 2e38)
        bias[-per:] = sign * 2e38 + 1e37
        check_route(l, bias.to(device()), 2, score, groups, 1, 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -3e38])
def test_finite_masks(mask, score):
    """experts masked by a large negative bias, of many and of most of them"""
    g = torch.Generator().manual_seed(3)
    l = torch.randn((37, 256), generator=g).to(device())
    bias = torch.randn((256,), generator=g) * 0.05
    for out in (3, 150, 252):
        b = bias.clone()
        b[torch.randperm(256, generator=g)[:out]] += mask
        b = b.to(device())
        check_route(l, b, 8, score)
        check_route(l, b, 8, score, 8, 4, 2)
        check_route(l, b, 8, score, 8, 4, 1, renorm=False)
