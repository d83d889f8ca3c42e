"""The model operators at the ends of their range."""
import math

import pytest
import torch

from tests import layer_util as lu
from tests import model_util as mu
from tests.gpu_util import device
from tests.test_gpu_router import check_route

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan


def oz():
    import paper_2606_06510_amd
    return paper_2606_06510_amd


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


# ------------------------------------------------------------------- loss

def exact_logits(z, T, dtype, K=16):
    """x and w whose logits are exactly the rows' z [V]: one product of 1 with z, zeros beside"""
    dt = lu.DTYPES[dtype]
    w = torch.zeros((z.numel(), K))
    w[:, K // 2] = z
    x = torch.zeros((T, K))
    x[:, K // 2] = 1.0
    assert torch.equal(w.to(dt).float(), w)
    return x.to(dt).to(device()), w.to(dt).to(device())


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,V", [(1, 1), (3, 40), (30, 700), (150, 900), (2048, 8192)])
def test_confident_tokens(T, V, dtype):
    """One word, or two, far above all others: a loss of 0 or log 2, whatever the logit's size.

    The sum of exponentials is 1 or 2, the others' share is below e^-40 V.  Off by: an
    exponential 2^-23, one for a chunk and one for the join, the sum and the logarithm
    2^-23 each, relative to a sum of 2 at most: 2^-20 in all, and the result's rounding."""
    sizes = [20.0, 100.0, 300.0, 1000.0]
    if dtype != "fp16":
        sizes += [2.0 ** 17, 1.5 * 2.0 ** 24, 1.25 * 2.0 ** 29, 1.75 * 2.0 ** 30, 2.0 ** 40, 3.0 * 2.0 ** 126]
    for size in sizes:
        for top in (size, -size):
            z = torch.full((V,), top - max(60.0, 2 * abs(top)) if abs(top) < 1e30 else -1.875 * 2.0 ** 127)
            z = z.to(lu.DTYPES[dtype]).float()
            z[V // 3] = top
            x, w = exact_logits(z, T, dtype)
            t = torch.full((T,), V // 3, device=device())
            loss, lse = oz().linear_cross_entropy(x, w, t)
            assert float(loss.abs().max()) <= 2.0 ** -20, (size, top, loss[0])
            assert float((lse.double() - top).abs().max()) <= 2.0 ** -20 + 2.0 ** -24 * abs(top)
            if V > 1:
                z[V - 1] = top
                x, w = exact_logits(z, T, dtype)
                loss, lse = oz().linear_cross_entropy(x, w, t)
                assert float((loss.double() - math.log(2)).abs().max()) <= 2.0 ** -20, (size, top, loss[0])


@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("T", [5, 40, 200, 4500])
def test_gradients_beside_one_that_is_no_number(T, value):
    """fp16: a counted token's dloss that is not finite leaves the others' rows of dX as they are.
    (Slopes are near 1e-8, below fp16's least number: without their power of two all would be 0.)"""
    g = torch.Generator().manual_seed(T)
    V, K = 3000, 64
    x = torch.randn((T, K), generator=g).half().to(device())
    w = (torch.randn((V, K), generator=g) * 0.1).half().to(device())
    t = torch.randint(0, V, (T,), generator=g).to(device())
    t[::9] = -1
    dl = ((0.5 + torch.rand((T,), generator=g)) * 1e-5).to(device())
    r = 2
    dl[r] = 4e-6                    # (not the largest, which gives the power of two)
    _, lse = oz().linear_cross_entropy(x, w, t)
    clean = oz().linear_cross_entropy_backward(dl, x, w, t, lse)
    assert float(clean[0][1].abs().max()) > 0
    d2 = dl.clone()
    d2[r] = value
    dx, dw = oz().linear_cross_entropy_backward(d2, x, w, t, lse)
    keep = torch.arange(T, device=x.device) != r
    assert torch.equal(dx[keep], clean[0][keep])
    assert not torch.isfinite(dx[r]).any() and not torch.isfinite(dw).any()
    only = torch.where(keep, torch.full_like(t, -1), t)      # the only one that counts
    dx, dw = oz().linear_cross_entropy_backward(d2, x, w, only, lse)
    assert (dx[keep] == 0).all() and not torch.isfinite(dx[r]).any()


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T", [2, 40, 150, 2048])
def test_infinite_logits(T, dtype):
    """lse = log sum e^z is infinite where a logit is, and the loss with it, but for a target
    whose own logit is infinite (no number)"""
    g = torch.Generator().manual_seed(T)
    dt = lu.DTYPES[dtype]
    V, K = 900 if T < 2048 else 8192, 64
    x, w = torch.randn((T, K), generator=g), torch.randn((V, K), generator=g) * 0.2
    x[:, 3] = x[:, 3].abs() + 0.5
    x[T - 1, 3] *= -1.0            # the last row has the logit -infinity
    t = torch.randint(0, V, (T,), generator=g)
    bad = 450
    t[t == bad] = 451
    if T > 2:
        t[1] = bad
    x, w, t = x.to(dt).to(device()), w.to(dt).to(device()), t.to(device())
    w[bad] = 0.0
    w[bad, 3] = INF
    clean = mu.loss(x[T - 1:], torch.cat([w[:bad], w[bad + 1:]]), t[T - 1:] - (t[T - 1:] > bad).long())
    loss, lse = oz().linear_cross_entropy(x, w, t)
    assert (lse[:T - 1] == INF).all()
    hit = t[:T - 1] == bad
    assert torch.isnan(loss[:T - 1][hit]).all() and (loss[:T - 1][~hit] == INF).all()
    lu.check(lse[T - 1:], clean[1], clean[3], "lse")
    lu.check(loss[T - 1:], clean[0], clean[2], "loss")
    w[bad + 9] = w[bad]            # and in another chunk's sums, and NaN over all
    w[7] = w[bad]
    loss, lse = oz().linear_cross_entropy(x, w, t)
    assert (lse[:T - 1] == INF).all()
    w[8, 3] = NAN
    loss, lse = oz().linear_cross_entropy(x, w, t)
    assert torch.isnan(lse).all() and torch.isnan(loss).all()


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T", [1, 3, 64, 65, 300])
def test_infinite_gradients(T, dtype):
    """an infinite dloss: the slopes are infinities of both signs, and so are the sums where
    none meets another sign's, or a zero"""
    dt, K = lu.DTYPES[dtype], 24
    g = torch.Generator().manual_seed(T)
    x = (torch.rand((T, K), generator=g) * 0.2 + 0.1).to(dt).to(device())
    w = torch.stack([torch.full((K,), 0.25), torch.full((K,), -0.5)]).to(dt).to(device())
    t = torch.ones(T, dtype=torch.int64, device=device())
    dl = torch.full((T,), 1e-3, device=device())
    _, lse = oz().linear_cross_entropy(x, w, t)
    clean = oz().linear_cross_entropy_backward(dl, x, w, t, lse)
    for sign in (1.0, -1.0):
        dl[0] = sign * INF
        dx, dw = oz().linear_cross_entropy_backward(dl, x, w, t, lse)
        # dz = (p, p' - 1) dloss = (+, -) infinity; dX = dz W, dW = dz^T x
        assert (dx[0] == sign * INF).all()
        assert (dw[0] == sign * INF).all() and (dw[1] == -sign * INF).all()
        if dtype != "fp16":        # (fp16: the power of two is that of the finite ones)
            assert torch.equal(dx[1:], clean[0][1:])


# ------------------------------------------------------------------- norm

def test_rows_of_no_width():
    """the mean and variance of nothing are 0 / 0"""
    for stream in (None, torch.cuda.current_stream()):
        for dtype in lu.DTYPES.values():
            x = torch.ones((6, 8), dtype=dtype, device=device())[:, :0]
            torch.full((4096,), 7.0, device=device())       # (freed memory that holds numbers)
            y, stats = oz().layer_norm(x, save_stats=True, stream=stream)
            assert y.shape == (6, 0) and stats.shape == (6, 2) and torch.isnan(stats).all()
            got = oz().layer_norm_backward(x, x, stats, stream=stream)
            assert got[0].shape == (6, 0) and got[1].shape == got[2].shape == (0,)
            y, stats = oz().layer_norm(x[:0], save_stats=True, stream=stream)
            assert stats.shape == (0, 2)
