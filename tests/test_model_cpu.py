"""The model operators without a GPU: the header's entry points are exported and bound,
arguments that the kernels could not take are refused before any launch (by the C ABI and by
the tensor helpers), and the plain forms of the GPU tests agree with each other."""
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2606_06510_amd as oz
from paper_2606_06510_amd import _lib
from tests import model_util as mu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MB = 1 << 20
AT = 1 << 40      # addresses that are never read: validation comes before any launch
BAD, SPACE = _lib.OZ2_E_INVALID, _lib.OZ2_E_WORKSPACE


def test_every_declared_entry_point_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "ozaki2", "model.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(ozaki2_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(_lib.MODEL_EXPORTS)
    for n in names:
        assert getattr(oz.load(), n).argtypes is not None and callable(getattr(oz, n))


ROUTE = dict(dtype=oz.OZ2_BF16, T=4, E=8, k=2, logits=AT, ld=8, bias=AT + MB, score=1, groups=4, top=2,
             best=2, renorm=1, scale=1.0, ids=AT + 2 * MB, w=AT + 3 * MB, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(dtype=-1), dict(T=-1), dict(E=0), dict(E=1025, ld=1025), dict(k=0), dict(k=5),
    dict(k=65, E=128, ld=128), dict(T=1 << 30), dict(logits=None), dict(logits=AT + 1), dict(ld=7),
    dict(bias=AT + MB + 2), dict(score=2), dict(score=-1), dict(groups=0), dict(groups=3),
    dict(groups=16), dict(top=0), dict(top=5), dict(best=0), dict(best=3), dict(ids=None),
    dict(ids=AT + 2 * MB + 1), dict(w=None), dict(w=AT + 2 * MB + 4), dict(ids=AT + 60), dict(w=AT + MB),
], ids=str)
def test_route_refusals(over):
    assert oz.load().ozaki2_expert_route(*{**ROUTE, **over}.values()) == BAD


BACK = dict(dtype=oz.OZ2_F16, T=4, E=8, k=2, dw=AT, logits=AT + MB, ld=8, ids=AT + 2 * MB, score=0,
            renorm=1, scale=1.0, dl=AT + 3 * MB, ldd=8, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(T=-1), dict(E=0), dict(E=1025, ld=1025, ldd=1025), dict(k=9), dict(k=0),
    dict(dw=None), dict(dw=AT + 2), dict(logits=None), dict(ld=7), dict(ids=None), dict(score=2),
    dict(dl=None), dict(dl=AT + 3 * MB + 1), dict(ldd=7), dict(dl=AT + MB), dict(dl=AT),
    dict(dl=AT + 2 * MB),
], ids=str)
def test_route_backward_refusals(over):
    assert oz.load().ozaki2_expert_route_backward(*{**BACK, **over}.values()) == BAD


NORM = dict(dtype=oz.OZ2_F32, T=4, K=6, x=AT, ldx=6, w=AT + MB, b=AT + 2 * MB, eps=1e-5, y=AT + 3 * MB,
            ldy=6, stats=AT + 4 * MB, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(T=-1), dict(K=-1), dict(K=(1 << 21) + 1), dict(T=1 << 30, K=1 << 10), dict(x=None),
    dict(x=AT + 2), dict(ldx=5), dict(w=AT + MB + 1), dict(b=AT + 2 * MB + 2), dict(eps=-1.0),
    dict(eps=math.nan), dict(y=None), dict(ldy=5), dict(y=AT + 4), dict(y=AT, ldy=7), dict(y=AT + MB),
    dict(y=AT + 2 * MB), dict(stats=AT + 3 * MB), dict(stats=AT), dict(stats=AT + 4 * MB + 1),
    dict(stats=AT + MB + 8),
], ids=str)
def test_norm_refusals(over):
    assert oz.load().ozaki2_layer_norm(*{**NORM, **over}.values()) == BAD


NORM_BACK = dict(dtype=oz.OZ2_F32, T=4, K=6, dy=AT, lddy=6, x=AT + MB, ldx=6, stats=AT + 2 * MB,
                 w=AT + 3 * MB, res=AT + 4 * MB, ldr=6, dx=AT + 5 * MB, lddx=6, dw=AT + 6 * MB,
                 db=AT + 7 * MB, ws=AT + 8 * MB, wsb=MB, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(T=-1), dict(K=-1), dict(dy=None), dict(lddy=5), dict(x=None), dict(ldx=5),
    dict(stats=None), dict(stats=AT + 2 * MB + 1), dict(w=AT + 3 * MB + 1), dict(ldr=5),
    dict(res=AT + 5 * MB + 4), dict(res=AT + 5 * MB, ldr=7), dict(dx=AT), dict(dx=AT + MB),
    dict(dx=AT + 2 * MB), dict(dx=AT + 3 * MB), dict(lddx=5), dict(dw=AT), dict(dw=AT + 5 * MB),
    dict(db=AT + 6 * MB + 8), dict(db=AT + 4 * MB), dict(dw=AT + 8 * MB), dict(dx=AT + 8 * MB),
    dict(stats=AT + 8 * MB),
], ids=str)
def test_norm_backward_refusals(over):
    assert oz.load().ozaki2_layer_norm_backward(*{**NORM_BACK, **over}.values()) == BAD


def test_norm_backward_workspace():
    need = oz.ozaki2_layer_norm_backward_workspace_bytes(oz.OZ2_F32, 4, 6)
    assert need >= 2 * 6 * 4
    L = oz.load()
    for over in (dict(ws=None), dict(wsb=need - 1), dict(ws=AT + 8 * MB + 64)):
        assert L.ozaki2_layer_norm_backward(*{**NORM_BACK, **over}.values()) == SPACE
    assert oz.ozaki2_layer_norm_backward_workspace_bytes(3, 4, 6) == 0


LOSS = dict(dtype=oz.OZ2_BF16, T=4, V=9, K=8, x=AT, ldx=8, w=AT + MB, ldw=8, t=AT + 2 * MB, wide=1,
            loss=AT + 3 * MB, lse=AT + 4 * MB, ws=AT + 5 * MB, wsb=MB, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(T=-1), dict(V=-1), dict(K=-1), dict(V=(1 << 21) + 1), dict(K=(1 << 21) + 1),
    dict(x=None), dict(x=AT + 1), dict(ldx=7), dict(w=None), dict(ldw=7), dict(t=None),
    dict(t=AT + 2 * MB + 4), dict(loss=None), dict(lse=None), dict(loss=AT + 3 * MB + 2),
    dict(lse=AT + 3 * MB + 8), dict(loss=AT), dict(lse=AT + MB), dict(loss=AT + 2 * MB), dict(ws=AT),
    dict(ws=AT + 4 * MB),
], ids=str)
def test_loss_refusals(over):
    assert oz.load().ozaki2_linear_cross_entropy(*{**LOSS, **over}.values()) == BAD


LOSS_BACK = dict(dtype=oz.OZ2_BF16, T=4, V=9, K=8, dl=AT, x=AT + MB, ldx=8, w=AT + 2 * MB, ldw=8,
                 t=AT + 3 * MB, wide=0, lse=AT + 4 * MB, dx=AT + 5 * MB, lddx=8, dw=AT + 6 * MB, lddw=8,
                 ws=AT + 7 * MB, wsb=MB, s=None)


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(T=-1), dict(V=-1), dict(K=-1), dict(dl=None), dict(dl=AT + 2), dict(x=None),
    dict(ldx=7), dict(w=None), dict(ldw=7), dict(t=None), dict(t=AT + 3 * MB + 2), dict(lse=None),
    dict(dx=AT + 1), dict(lddx=7), dict(lddw=7), dict(dx=AT), dict(dx=AT + MB), dict(dw=AT + 2 * MB),
    dict(dw=AT + 3 * MB), dict(dx=AT + 4 * MB), dict(dw=AT + 5 * MB + 16), dict(ws=AT + MB),
    dict(ws=AT + 6 * MB),
], ids=str)
def test_loss_backward_refusals(over):
    assert oz.load().ozaki2_linear_cross_entropy_backward(*{**LOSS_BACK, **over}.values()) == BAD


def test_loss_workspaces():
    L = oz.load()
    need = oz.ozaki2_linear_cross_entropy_workspace_bytes(oz.OZ2_BF16, 4, 9, 8)
    for over in (dict(ws=None), dict(wsb=need - 1), dict(ws=AT + 5 * MB + 16)):
        assert L.ozaki2_linear_cross_entropy(*{**LOSS, **over}.values()) == SPACE
    need = oz.ozaki2_linear_cross_entropy_backward_workspace_bytes(oz.OZ2_BF16, 4, 9, 8)
    for over in (dict(ws=None), dict(wsb=need - 1), dict(ws=AT + 7 * MB + 16)):
        assert L.ozaki2_linear_cross_entropy_backward(*{**LOSS_BACK, **over}.values()) == SPACE
    assert oz.ozaki2_linear_cross_entropy_workspace_bytes(3, 4, 9, 8) == 0
    assert oz.ozaki2_linear_cross_entropy_backward_workspace_bytes(2, -4, 9, 8) == 0
    # the logits of a long batch are never there as a whole
    T, V, K = 65536, 131072, 4096
    for f in (oz.ozaki2_linear_cross_entropy_workspace_bytes,
              oz.ozaki2_linear_cross_entropy_backward_workspace_bytes):
        assert f(oz.OZ2_BF16, T, V, K) < T * V * 2 / 6


def test_nothing_to_do_is_no_error():
    L = oz.load()
    assert L.ozaki2_expert_route(*{**ROUTE, "T": 0, "logits": None}.values()) == 0
    assert L.ozaki2_expert_route_backward(*{**BACK, "T": 0, "dl": None}.values()) == 0
    assert L.ozaki2_layer_norm(*{**NORM, "T": 0, "x": None}.values()) == 0
    assert L.ozaki2_layer_norm(*{**NORM, "K": 0, "y": None}.values()) == 0
    assert L.ozaki2_layer_norm_backward(*{**NORM_BACK, "dx": None, "dw": None, "db": None}.values()) == 0
    assert L.ozaki2_linear_cross_entropy(*{**LOSS, "T": 0, "x": None}.values()) == 0
    assert L.ozaki2_linear_cross_entropy_backward(*{**LOSS_BACK, "dx": None, "dw": None}.values()) == 0


@pytest.fixture
def no_device(monkeypatch):
    """A tensor that claims to be on the GPU is not to be had here: the checks of types,
    shapes and strides come before or beside that of the device."""
    from paper_2606_06510_amd import model

    def boom(*a, **k):
        raise AssertionError("a library entry point was reached")
    for name in _lib.MODEL_EXPORTS:
        if not name.endswith("_bytes"):
            monkeypatch.setattr(_lib, name, boom)
    monkeypatch.setattr(model, "_device", lambda name, t: t.device)


def refuse(f, base, cases, error=ValueError):
    for over, match in cases:
        with pytest.raises(error, match=match):
            f(**{**base, **over})


def test_tensors_off_the_device():
    x = torch.zeros(4, 8)
    for call in (lambda: oz.expert_route(x, 2), lambda: oz.layer_norm(x),
                 lambda: oz.expert_route_backward(x, x, x), lambda: oz.layer_norm_backward(x, x, x),
                 lambda: oz.linear_cross_entropy(x, x, x),
                 lambda: oz.linear_cross_entropy_backward(x, x, x, x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_tensor_checks(no_device):
    x, f = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8)
    refuse(oz.expert_route, dict(logits=x, top_k=2), [
        (dict(logits=x.double()), "float32, float16 or bfloat16"), (dict(score="tanh"), "score"),
        (dict(top_k=0), "top_k"), (dict(top_k=9), "top_k"), (dict(groups=3), "groups"),
        (dict(groups=0), "groups"), (dict(groups=4, top_groups=5), "top_groups"),
        (dict(groups=4, top_groups=1, top_k=3), "top_k"), (dict(group_best=3), "group_best"),
        (dict(bias=x[0]), "dtype"), (dict(bias=f[:7]), "shape"), (dict(logits=x[0]), "dimensions"),
        (dict(bias=torch.zeros(16)[::2]), "contiguous"), (dict(logits=x.t()), "adjacent"),
        (dict(logits=torch.zeros(2, 1025)), "experts")])
    ids, dw = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    refuse(oz.expert_route_backward, dict(dweights=dw, logits=x, ids=ids), [
        (dict(ids=ids.long()), "dtype"), (dict(ids=ids[:3]), "tokens"), (dict(dweights=dw.half()), "dtype"),
        (dict(dweights=dw[:, :1]), "shape"), (dict(score=None), "score"), (dict(dlogits=x[:, :7]), "shape"),
        (dict(dlogits=x.float()), "dtype"), (dict(ids=torch.zeros(4, 9, dtype=torch.int32)), "top_k")])
    w, stats = x[0], torch.zeros(4, 2)
    refuse(oz.layer_norm, dict(x=x), [
        (dict(weight=f), "dtype"), (dict(weight=w[:7]), "shape"), (dict(bias=x), "shape"), (dict(eps=-1.0), "eps"),
        (dict(eps=math.nan), "eps"), (dict(out=x[:3]), "shape"), (dict(x=x.t()), "adjacent"),
        (dict(out=x.float()), "dtype"), (dict(x=x[:1].expand(4, 8)), "overlap")])
    refuse(oz.layer_norm_backward, dict(dy=x, x=x, stats=stats), [
        (dict(x=x[:3]), "shape"), (dict(stats=stats[:3]), "shape"), (dict(stats=stats.half()), "dtype"),
        (dict(weight=f), "dtype"), (dict(residual=x.float()), "dtype"), (dict(dx=x[:, :7]), "shape"),
        (dict(dweight=w[:5]), "shape"), (dict(dbias=f), "dtype"), (dict(stats=torch.zeros(2, 4).t()),
                                                                   "contiguous")])
    v, t = torch.zeros(9, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    refuse(oz.linear_cross_entropy, dict(x=x, w=v, targets=t), [
        (dict(w=v[:, :7]), "shape"), (dict(w=v.float()), "dtype"), (dict(targets=t[:3]), "shape"),
        (dict(targets=t.float()), "int32 or int64"), (dict(targets=torch.zeros(8, dtype=torch.int64)[::2]),
                                                      "contiguous"), (dict(w=v.t()), "shape|adjacent")])
    s = torch.zeros(4)
    refuse(oz.linear_cross_entropy_backward, dict(dloss=s, x=x, w=v, targets=t, lse=s), [
        (dict(dloss=s.half()), "dtype"), (dict(lse=s[:3]), "shape"), (dict(dx=x[:3]), "shape"),
        (dict(dw=v.float()), "dtype"), (dict(targets=t.short()), "int32 or int64"), (dict(w=v[0]), "dimensions")])


@pytest.mark.parametrize("wrong", [None, 3, [[1.0]], np.zeros((4, 8), np.float32)],
                         ids=["None", "number", "list", "array"])
def test_no_tensor(wrong, no_device):
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    ids, s = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4)
    calls = {"logits": [lambda: oz.expert_route(wrong, 2), lambda: oz.expert_route_backward(x, wrong, ids)],
             "ids": [lambda: oz.expert_route_backward(x[:, :2].contiguous(), x, wrong)],
             "dweights": [lambda: oz.expert_route_backward(wrong, x, ids)],
             "x": [lambda: oz.layer_norm(wrong), lambda: oz.linear_cross_entropy(wrong, x, t),
                   lambda: oz.layer_norm_backward(x, wrong, x[:, :2].contiguous())],
             "dy": [lambda: oz.layer_norm_backward(wrong, x, ids)],
             "stats": [lambda: oz.layer_norm_backward(x, x, wrong)],
             "w": [lambda: oz.linear_cross_entropy(x, wrong, t)],
             "targets": [lambda: oz.linear_cross_entropy(x, x, wrong)],
             "dloss": [lambda: oz.linear_cross_entropy_backward(wrong, x, x, t, s)],
             "lse": [lambda: oz.linear_cross_entropy_backward(s, x, x, t, wrong)]}
    for name, some in calls.items():
        for call in some:
            with pytest.raises(TypeError, match=f"{name}: expected a torch tensor"):
                call()


class Doubtful:
    def __bool__(self):
        raise ValueError("neither")


def test_the_short_path_leaves_everything_else_to_the_other():
    """tensors elsewhere, arguments of other types and numbers of arguments: None, and no exception"""
    from paper_2606_06510_amd import model
    f = model._bind()
    x, ids, dw = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for wrong in (None, 3, "x", [1.0], np.zeros((4, 8), np.float32), x, x.to_sparse(), x.t(),
                  torch.nn.Parameter(x), torch.zeros(4, 8, device="meta")):
        assert f.layer_norm(wrong, None, None, 1e-5, False) is None
        assert f.expert_route(wrong, 2, None, 0, 1, 1, 1, True, 1.0) is None
        assert f.expert_route_backward(dw, wrong, ids, 0, True, 1.0) is None
        assert f.expert_route_backward(wrong, x, ids, 0, True, 1.0) is None
        t = torch.zeros(4, dtype=torch.int64)
        assert f.layer_norm_backward(wrong, x, dw, None, None, True, True, True) is None
        assert f.linear_cross_entropy(x, wrong, t) is None
        assert f.linear_cross_entropy_backward(x[0], x, wrong, t, x[0], True, True) is None
    assert f.layer_norm_backward() is None and f.linear_cross_entropy() is None
    assert f.linear_cross_entropy_backward(None) is None
    assert f.layer_norm() is None and f.expert_route(x) is None and f.expert_route_backward() is None
    assert f.layer_norm(x, None, None, "eps", False) is None
    assert f.expert_route(x, 1 << 80, None, 0, 1, 1, 1, True, 1.0) is None
    assert f.expert_route(x, 2, None, 0, 1, 1, 1, Doubtful(), 1.0) is None
    assert f.expert_route(x, 2, None, 0, 1, 1, 1, True, 1 << 2000) is None
    with pytest.raises(TypeError):
        f.bind(1)


# -------------------------------------------------- the plain forms agree with autograd

@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_plain_router_gradient(score, renorm):
    """by differences of the plain weights, the choice held"""
    g = torch.Generator().manual_seed(3)
    l = torch.randn((1, 6), generator=g, dtype=torch.float64)
    dw = torch.randn((1, 3), generator=g, dtype=torch.float64)
    ids, _ = mu.route_row(l[0].tolist(), None, 3, score, 1, 1, 1, renorm, 1.5)
    got = mu.route_backward(dw, l, torch.tensor([ids]), score, renorm, 1.5)[0]

    def value(row):
        i, w = mu.route_row(row.tolist(), None, 3, score, 1, 1, 1, renorm, 1.5)
        assert i == ids
        return sum(a * b for a, b in zip(w, dw[0].tolist()))
    for e in range(6):
        h = torch.zeros(6, dtype=torch.float64)
        h[e] = 1e-6
        slope = (value(l[0] + h) - value(l[0] - h)) / 2e-6
        assert abs(slope - float(got[e])) < 1e-8


def test_plain_norm_gradient():
    g = torch.Generator().manual_seed(4)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64).requires_grad_(True)
                   for s in ((5, 7), (7,), (7,), (5, 7)))
    y = torch.nn.functional.layer_norm(x, (7,), w, b, 1e-5)
    want = torch.autograd.grad((y * dy.detach()).sum(), (x, w, b))
    ref = mu.norm(x, w, b, 1e-5)
    assert torch.allclose(ref[0], y.detach(), rtol=1e-12, atol=1e-12)
    for a, c in zip(mu.norm_backward(dy, x, ref[1], w, None)[:3], want):
        assert torch.allclose(a, c, rtol=1e-10, atol=1e-12)


def test_plain_loss_gradient():
    g = torch.Generator().manual_seed(5)
    x, w = (torch.randn(s, generator=g, dtype=torch.float64).requires_grad_(True) for s in ((6, 4), (9, 4)))
    t, dl = torch.tensor([0, 8, -100, 3, 9, 5]), torch.rand((6,), generator=g, dtype=torch.float64)
    t9 = torch.where(t == 9, -100, t)
    per = torch.nn.functional.cross_entropy(x @ w.t(), t9, ignore_index=-100, reduction="none")
    want = torch.autograd.grad((per * dl).sum(), (x, w))
    loss, lse = mu.loss(x, w, t)[:2]
    assert torch.allclose(loss, per.detach(), rtol=1e-12, atol=1e-12)
    got = mu.loss_backward(dl, x, w, t, lse, torch.float32)
    for a, c in zip(got[:2], want):
        assert torch.allclose(a, c, rtol=1e-10, atol=1e-12)
