"""linear_cross_entropy and its gradients against 64-bit forms."""
import math

import pytest
import torch

from tests import layer_util as lu
from tests import model_util as mu
from tests.gpu_util import device

pytestmark = pytest.mark.gpu


def oz():
    import paper_2606_06510_amd
    return paper_2606_06510_amd


@pytest.fixture(autouse=True)
def on_gpu(monkeypatch):
    monkeypatch.setattr(lu, "ON_GPU", True)    # the 64-bit products


def make(T, V, K, dtype, seed, ignore=0.2, wide=True, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    dt = lu.DTYPES[dtype]
    x = torch.randn((T, K), generator=g).to(dt)
    w = (torch.randn((V, K), generator=g) * scale * max(K, 1) ** -0.5).to(dt)
    t = torch.randint(0, max(V, 1), (T,), generator=g)
    t[torch.rand((T,), generator=g) < ignore] = -100
    dl = torch.rand((T,), generator=g) / max(T, 1)
    return dict(x=x.to(device()), w=w.to(device()), t=(t if wide else t.int()).to(device()), dl=dl.to(device()))


def check_loss(c):
    loss, lse = oz().linear_cross_entropy(c["x"], c["w"], c["t"])
    assert loss.dtype == lse.dtype == torch.float32
    want = mu.loss(c["x"], c["w"], c["t"])
    lu.check(lse, want[1], want[3], "lse")
    lu.check(loss, want[0], want[2], "loss")
    return loss, lse


def check_grad(c, lse, **kw):
    got = oz().linear_cross_entropy_backward(c["dl"], c["x"], c["w"], c["t"], lse, **kw)
    want = mu.loss_backward(c["dl"], c["x"], c["w"], c["t"], lse, c["x"].dtype)
    for name, a, r, e in zip(("dx", "dw"), got, want[:2], want[2:]):
        if a is not None:
            lu.check(a, r, e, name)
    return got


SIZES = [(1, 1, 1), (1, 5, 8), (2, 16, 64), (3, 17, 72), (5, 100, 40), (16, 1000, 128), (17, 33, 256), (32, 777, 200),
         (33, 300, 64), (64, 4096, 128), (100, 1001, 333), (130, 515, 96), (257, 2049, 72), (300, 10, 512),
         (700, 3000, 136), (1, 50021, 64), (4, 20000, 1024), (40, 9, 2000)]


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,V,K", SIZES)
def test_loss_and_gradients(T, V, K, dtype):
    c = make(T, V, K, dtype, T + V + K, wide=T % 2 == 0)
    loss, lse = check_loss(c)
    check_grad(c, lse)


@pytest.mark.parametrize("dtype,T,V,K", [("bf16", 2048, 8192, 512), ("fp16", 1500, 7001, 1024),
                                         ("bf16", 4100, 5000, 264), ("fp32", 1030, 4100, 260),
                                         ("bf16", 3000, 2049, 1001), ("fp16", 600, 40000, 64)])
def test_large_tiles(dtype, T, V, K):
    """sizes that take 256 wide tiles, odd ends of each dimension"""
    c = make(T, V, K, dtype, T)
    loss, lse = check_loss(c)
    again = oz().linear_cross_entropy(c["x"], c["w"], c["t"])
    assert torch.equal(loss, again[0]) and torch.equal(lse, again[1])
    a = check_grad(c, lse)
    b = oz().linear_cross_entropy_backward(c["dl"], c["x"], c["w"], c["t"], lse)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def pieces(T, V, K, dtype):
    """words of a piece: 128 MiB of slopes"""
    e = 4 if dtype == "fp32" else 2
    return min(V, max(256, (128 << 20) // e // T // 256 * 256))


@pytest.mark.parametrize("dtype,T,V,K", [("bf16", 9000, 40001, 72), ("fp16", 20000, 16000, 64),
                                         ("fp32", 5000, 30003, 36)])
def test_pieces_of_the_vocabulary(dtype, T, V, K):
    """gradients in more than one piece, the last one short"""
    assert pieces(T, V, K, dtype) < V and V % pieces(T, V, K, dtype)
    c = make(T, V, K, dtype, 7)
    loss, lse = check_loss(c)
    check_grad(c, lse)


def test_pieces_of_the_rows():
    """more rows than the chunks of one launch hold: half a GiB"""
    T, V = 8400, 524300
    c = make(T, V, 8, "bf16", 9)
    full = oz().linear_cross_entropy(c["x"], c["w"], c["t"])
    for r in (0, 4000, 8192, 8390):
        part = {k: v if k == "w" else v[r:r + 10] for k, v in c.items()}
        want = mu.loss(part["x"], part["w"], part["t"])
        lu.check(full[1][r:r + 10], want[1], want[3], "lse")
        lu.check(full[0][r:r + 10], want[0], want[2], "loss")


def test_every_target_of_a_tile_and_none():
    """each word once (all chunks, lanes and columns hold a target), targets at and outside the
    ends, of both types"""
    V, K = 600, 64
    for wide in (True, False):
        c = make(V + 6, V, K, "bf16", 3, ignore=0.0)
        t = torch.arange(V + 6)
        t[V:] = torch.tensor([-1, V, V + 7, -100, 2 ** 31 - 1, -2 ** 31])
        c["t"] = (t if wide else t.int()).to(device())
        loss, lse = check_loss(c)
        assert (loss[V:] == 0).all() and (loss[:V] != 0).all()
        dx, _ = check_grad(c, lse)
        assert (dx[V:] == 0).all()
    c["t"] = torch.full((V + 6,), 2 ** 40, dtype=torch.int64, device=device())   # none counts
    loss, lse = check_loss(c)
    dx, dw = check_grad(c, lse)
    assert (loss == 0).all() and (dx == 0).all() and (dw == 0).all()
    for T in (4, 40):   # the kernels of few rows and of small tiles
        d = make(T, 70, K, "fp32", T, ignore=0.0)
        for r in range(0, 70, T):
            d["t"] = (torch.arange(r, r + T)).to(device())
            _, lse = check_loss(d)
            check_grad(d, lse)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T", [6, 90, 600])
def test_rows_that_do_not_count_hold_anything(T, dtype):
    c = make(T, 700, 136, dtype, T)
    loss, lse = check_loss(c)
    clean = check_grad(c, lse)
    off = c["t"] < 0
    assert off.any() and not off.all()
    c["x"][off] = math.nan
    dl, l2 = c["dl"].clone(), lse.clone()
    dl[off], l2[off] = math.inf, math.nan
    got = oz().linear_cross_entropy(c["x"], c["w"], c["t"])
    assert torch.equal(got[0], loss) and torch.equal(got[1][~off], lse[~off])
    got = oz().linear_cross_entropy_backward(dl, c["x"], c["w"], c["t"], l2)
    assert all(torch.equal(a, b) for a, b in zip(got, clean)) and (got[0][off] == 0).all()


@pytest.mark.parametrize("T", [5, 70])
def test_infinities_and_nan(T):
    c = make(T, 300, 64, "fp32", T, ignore=0.0)
    loss, lse = check_loss(c)
    x = c["x"].clone()
    x[2, 5] = math.nan
    got = oz().linear_cross_entropy(x, c["w"], c["t"])
    keep = torch.arange(T) != 2
    assert torch.isnan(got[0][2]) and torch.isnan(got[1][2])
    assert torch.equal(got[0][keep], loss[keep]) and torch.equal(got[1][keep], lse[keep])
    w = c["w"].clone()
    w[7] = 0.0
    w[7, 0] = -math.inf          # a word that is never meant: its logit is -infinity where x[0] > 0
    x = c["x"].clone()
    x[:, 0] = x[:, 0].abs() + 0.5
    d = dict(c, x=x, w=w, t=torch.where(c["t"] == 7, 8, c["t"]))
    rest = dict(d, w=torch.cat([w[:7], w[8:]]), t=torch.where(d["t"] > 7, d["t"] - 1, d["t"]))
    want = mu.loss(rest["x"], rest["w"], rest["t"])
    got = oz().linear_cross_entropy(d["x"], d["w"], d["t"])
    lu.check(got[1], want[1], want[3], "lse")
    lu.check(got[0], want[0], want[2], "loss")


def test_large_logits():
    """a spread of hundreds: no exponential of a large number"""
    for T in (3, 200):
        c = make(T, 1000, 64, "fp32", 4, scale=400.0)
        loss, lse = check_loss(c)
        assert float(lse.max()) > 500
        check_grad(c, lse)


def test_small_gradients_in_fp16():
    """slopes far below fp16's range, and large ones: scaled on their way to the products"""
    for T, f in ((50, 1e-6), (50, 1e-9), (600, 3e-7), (50, 1e4), (4, 1e-20)):
        c = make(T, 2000, 72, "fp16", 8)
        c["dl"] *= f * T
        loss, lse = check_loss(c)
        big = dict(c, w=c["w"], dl=c["dl"])
        got = check_grad(big, lse)
        if f >= 1e-6:
            assert float(got[1].abs().max()) > 0


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T", [7, 150])
def test_strided_unaligned_and_given_outputs(T, dtype):
    V, K = 530, 88
    c = make(T, V, K, dtype, T)
    loss, lse = check_loss(c)
    grads = check_grad(c, lse)

    def view(t, at):
        big = torch.full((t.shape[0], K + 11), 9.0, dtype=t.dtype, device=t.device)
        v = big[:, at:at + K]
        v.copy_(t)
        return big, v
    bx, x = view(c["x"], 3)
    bw, w = view(c["w"], 5)
    d = dict(c, x=x, w=w)
    check_loss(d)
    bdx, dx = view(c["x"], 1)
    bdw, dw = view(c["w"], 7)
    got = check_grad(d, lse, dx=dx, dw=dw)
    assert got[0] is dx and got[1] is dw
    for big, at in ((bdx, 1), (bdw, 7)):
        assert (big[:, :at] == 9).all() and (big[:, at + K:] == 9).all()
    one = oz().linear_cross_entropy_backward(c["dl"], c["x"], c["w"], c["t"], lse, need_dw=False)
    two = oz().linear_cross_entropy_backward(c["dl"], c["x"], c["w"], c["t"], lse, need_dx=False)
    assert torch.equal(one[0], grads[0]) and one[1] is None
    assert torch.equal(two[1], grads[1]) and two[0] is None


def test_empty_sizes():
    c = make(5, 40, 16, "bf16", 1)
    assert oz().linear_cross_entropy(c["x"][:0], c["w"], c["t"][:0])[0].shape == (0,)
    dx, dw = oz().linear_cross_entropy_backward(c["dl"][:0], c["x"][:0], c["w"], c["t"][:0], c["dl"][:0])
    assert dx.shape == (0, 16) and (dw == 0).all()
    loss, lse = oz().linear_cross_entropy(c["x"], c["w"][:0], c["t"])
    assert (loss == 0).all() and (lse == -math.inf).all()
    dx, dw = oz().linear_cross_entropy_backward(c["dl"], c["x"], c["w"][:0], c["t"], lse)
    assert (dx == 0).all() and dw.shape == (0, 16)
    loss, lse = oz().linear_cross_entropy(c["x"][:, :0], c["w"][:, :0], c["t"])     # logits of 0
    assert torch.allclose(lse, torch.full_like(lse, math.log(40)))
    dx, dw = oz().linear_cross_entropy_backward(c["dl"], c["x"][:, :0], c["w"][:, :0], c["t"], lse)
    assert dx.shape == (5, 0) and dw.shape == (40, 0)


@pytest.mark.parametrize("T", [3, 60])
def test_gradient_by_differences(T):
    """fp32: the loss's change along a direction"""
    c = make(T, 90, 24, "fp32", 5, scale=1.0)
    dl = c["dl"]
    _, lse = check_loss(c)
    dx, dw = check_grad(c, lse)
    g = torch.Generator().manual_seed(6)
    for name, grad in (("x", dx), ("w", dw)):
        v = torch.randn(c[name].shape, generator=g).to(device())

        def at(h):
            loss = mu.loss(*(c[n] if n != name else c[n].double() + h * v.double() for n in ("x", "w", "t")))[0]
            return float((loss * dl.double()).sum())
        h = 1e-5
        slope = (at(h) - at(-h)) / (2 * h)
        total = float((grad.double() * v.double()).sum())
        # the gradient's own rounding, and h^2 of the third derivative
        assert abs(slope - total) < 1e-5 * float((grad.double() * v.double()).abs().sum()) + 1e-8
