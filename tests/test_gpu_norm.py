"""layer_norm and its gradients against 64-bit forms."""
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


def make(T, K, dtype, seed, shift=0.5, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    dt = lu.DTYPES[dtype]

    def normal(*shape, s=1.0, m=0.0):
        return (torch.randn(shape, generator=g) * s + m).to(dt).to(device())
    return dict(x=normal(T, K, s=spread, m=shift), w=normal(K, s=0.3, m=1.0), b=normal(K, s=0.3),
                dy=normal(T, K), r=normal(T, K))


def check_norm(x, w, b, eps=1e-5):
    y, stats = oz().layer_norm(x, w, b, eps=eps, save_stats=True)
    want, ws, ey, es = mu.norm(x, w, b, eps)
    lu.check(stats, ws, es, "stats")
    lu.check(y, want, ey, "y")
    assert torch.equal(y, oz().layer_norm(x, w, b, eps=eps))
    return y, stats


def check_back(dy, x, stats, w, r, **kw):
    got = oz().layer_norm_backward(dy, x, stats, weight=w, residual=r, **kw)
    want = mu.norm_backward(dy, x, stats, w, r)
    for name, a, c, e in zip(("dx", "dweight", "dbias"), got, want[:3], want[3:]):
        if a is not None:
            lu.check(a, c, e, name)
    return got


SIZES = [(1, 1), (1, 2), (3, 7), (2, 64), (65, 63), (5, 100), (300, 129), (17, 512), (4, 1000), (33, 1024),
         (9, 1203), (2, 2001), (70, 2048), (3, 4095), (6, 4096), (2, 4104), (3, 8192), (2, 8200), (2, 12345),
         (3, 16384), (2, 16392), (2, 20001), (1, 70001)]


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,K", SIZES)
def test_rows(T, K, dtype):
    c = make(T, K, dtype, T + K)
    check_norm(c["x"], c["w"], c["b"])
    check_norm(c["x"], c["w"], None, eps=1e-3)
    _, stats = check_norm(c["x"], None, None)
    check_back(c["dy"], c["x"], stats, c["w"], c["r"])
    check_back(c["dy"], c["x"], stats, None, None)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,K", [(5000, 96), (1111, 1203), (3000, 4096), (16400, 64), (700, 8192), (260, 16500),
                                 (70000, 8), (40000, 1)])
def test_many_rows(T, K, dtype):
    c = make(T, K, dtype, T + K)
    y, stats = check_norm(c["x"], c["w"], c["b"])
    a = check_back(c["dy"], c["x"], stats, c["w"], c["r"])
    b = oz().layer_norm_backward(c["dy"], c["x"], stats, weight=c["w"], residual=c["r"])
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("K", [64, 1203, 4096, 9000])
def test_each_gradient_alone(K):
    c = make(300, K, "bf16", K)
    _, stats = check_norm(c["x"], c["w"], c["b"])
    full = check_back(c["dy"], c["x"], stats, c["w"], None)
    for i in range(3):
        need = dict(zip(("need_dx", "need_dweight", "need_dbias"), (i == 0, i == 1, i == 2)))
        got = oz().layer_norm_backward(c["dy"], c["x"], stats, weight=c["w"], **need)
        assert torch.equal(got[i], full[i]) and all(got[j] is None for j in range(3) if j != i)
    two = oz().layer_norm_backward(c["dy"], c["x"], stats, weight=c["w"], need_dbias=False)
    assert torch.equal(two[0], full[0]) and torch.equal(two[1], full[1]) and two[2] is None
    assert oz().layer_norm_backward(c["dy"], c["x"], stats, need_dx=False, need_dweight=False,
                                    need_dbias=False) == (None, None, None)


def test_constant_rows_and_rows_far_from_zero():
    """no variance: eps alone; a mean of 1000 beside a spread of 1 (the variance is taken about
    the mean)"""
    for dtype in lu.DTYPES:
        x = torch.full((3, 777), 1.25, dtype=lu.DTYPES[dtype], device=device())
        y, stats = check_norm(x, None, None)
        assert (y == 0).all()
        x[1] = 0.0
        check_norm(x, None, None)
    g = torch.Generator().manual_seed(1)
    x = (torch.randn((20, 1500), generator=g) + 1000.0).to(device())
    y, stats = check_norm(x, None, None)
    check_back(torch.randn((20, 1500), generator=g).to(device()), x, stats, None, None)
    x = torch.zeros((2, 33), device=device())
    y = oz().layer_norm(x, eps=0.0)
    assert torch.isnan(y).all()     # 0 / 0


@pytest.mark.parametrize("K", [40, 600, 5000])
def test_infinities_and_nan_stay_in_their_rows(K):
    c = make(9, K, "fp32", K)
    clean, st = check_norm(c["x"], c["w"], c["b"])
    x = c["x"].clone()
    x[2, 3], x[5, K - 1], x[7, 0] = math.nan, math.inf, -math.inf
    y, stats = oz().layer_norm(x, c["w"], c["b"], save_stats=True)
    for t in range(9):
        if t in (2, 5, 7):
            assert torch.isnan(y[t]).all()
        else:
            assert torch.equal(y[t], clean[t]) and torch.equal(stats[t], st[t])
    good = check_back(c["dy"], c["x"], st, c["w"], None)[0]
    dx, dw, db = oz().layer_norm_backward(c["dy"], x, stats, weight=c["w"])
    for t in range(9):
        assert torch.isnan(dx[t]).all() if t in (2, 5, 7) else torch.equal(dx[t], good[t])
    assert torch.isnan(dw).all() and not torch.isnan(db).any()


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("K", [24, 1001, 4096, 8200])
def test_strided_unaligned_and_in_place(K, dtype):
    c = make(37, K, dtype, K)

    def view(t, at):
        big = torch.full((t.shape[0], K + 13), 9.0, dtype=t.dtype, device=t.device)
        v = big[:, at:at + K]
        v.copy_(t)
        return big, v
    y, stats = check_norm(c["x"], c["w"], c["b"])
    grads = check_back(c["dy"], c["x"], stats, c["w"], c["r"])
    bx, x = view(c["x"], 3)
    bo, out = view(c["dy"], 5)
    wb = torch.empty(K + 1, dtype=c["w"].dtype, device=device())[1:]
    wb.copy_(c["w"])
    got = oz().layer_norm(x, wb, c["b"], out=out)
    assert got is out and torch.equal(out, y)
    assert (bo[:, :5] == 9).all() and (bo[:, 5 + K:] == 9).all()
    _, dy = view(c["dy"], 1)
    br, r = view(c["r"], 7)
    got = oz().layer_norm_backward(dy, x, stats, weight=wb, residual=r, dx=r)   # in place of the residual
    assert got[0] is r and all(torch.equal(a, b) for a, b in zip(got, grads))
    assert (br[:, :7] == 9).all() and (br[:, 7 + K:] == 9).all()
    got = oz().layer_norm(x, c["w"], c["b"], out=x)
    assert torch.equal(x, y) and (bx[:, :3] == 9).all() and (bx[:, 3 + K:] == 9).all()


def test_no_rows():
    c = make(4, 50, "bf16", 2)
    y, stats = oz().layer_norm(c["x"][:0], c["w"], save_stats=True)
    assert y.shape == (0, 50) and stats.shape == (0, 2)
    dx, dw, db = oz().layer_norm_backward(c["dy"][:0], c["x"][:0], stats, weight=c["w"])
    assert dx.shape == (0, 50) and (dw == 0).all() and (db == 0).all()
    assert oz().layer_norm(c["x"][:, :0]).shape == (4, 0)
