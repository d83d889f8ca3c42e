"""The layer operators without a GPU: the header's entry points are exported and
bound, arguments that the kernels could not take are refused before any launch
(by the C ABI and by the tensor helpers), and the plain forms of the GPU tests
agree with each other."""
import ctypes
import os
import re

import pytest
import torch

import paper_2606_06510_amd as oz
from paper_2606_06510_amd import _lib
from tests import layer_util as lu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MB = 1 << 20
AT = 1 << 40      # addresses that are never read: validation comes before any launch


def test_every_declared_entry_point_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "ozaki2", "layers.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(ozaki2_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(_lib.LAYER_EXPORTS) and len(names) == 13
    L = oz.load()
    for n in names:
        assert getattr(L, n).argtypes is not None and callable(getattr(oz, n))


def linear_args(**over):
    a = dict(dtype=oz.OZ2_BF16, act=oz.OZ2_ACT_SILU, gated=0, rows=4, out=6, inp=8, x=AT, ldx=8,
             w=AT + MB, ldw=8, bias=AT + 2 * MB, res=AT + 3 * MB, ldr=6, y=AT + 4 * MB, ldy=6,
             z=AT + 5 * MB, ldz=6, ws=AT + 6 * MB, wsb=MB, stream=None)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over", [
    dict(dtype=3), dict(dtype=-1), dict(act=5), dict(act=-1), dict(rows=-1), dict(out=-1),
    dict(inp=-1), dict(out=1 << 25), dict(rows=1 << 30, out=1 << 20), dict(x=None), dict(w=None),
    dict(y=None), dict(x=AT + 1), dict(y=AT + 4 * MB + 1), dict(bias=AT + 2 * MB + 1), dict(ldx=7),
    dict(ldw=7), dict(ldr=5), dict(ldy=5), dict(ldz=5), dict(ldx=1 << 41), dict(gated=1, ldz=11),
    dict(y=AT), dict(y=AT + MB), dict(y=AT + 2 * MB), dict(z=AT + 8), dict(z=AT + 4 * MB + 12),
    dict(res=AT + 4 * MB + 2), dict(res=AT + 4 * MB, ldr=7),
], ids=str)
def test_linear_refusals(over):
    assert oz.load().ozaki2_linear(*linear_args(**over)) == _lib.OZ2_E_INVALID


def backward_args(**over):
    a = dict(dtype=oz.OZ2_F16, act=oz.OZ2_ACT_GELU, gated=0, rows=4, out=6, inp=8, dy=AT, lddy=6,
             x=AT + MB, ldx=8, w=AT + 2 * MB, ldw=8, z=AT + 3 * MB, ldz=6, dx=AT + 4 * MB, lddx=8,
             dw=AT + 5 * MB, lddw=8, db=AT + 6 * MB, ws=AT + 7 * MB, wsb=MB, stream=None)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over", [
    dict(dtype=7), dict(act=9), dict(rows=-1), dict(dy=None), dict(x=None), dict(w=None),
    dict(z=None), dict(z=AT + 3 * MB + 1), dict(lddy=5), dict(ldx=7), dict(ldw=7), dict(ldz=5),
    dict(lddx=7), dict(lddw=7), dict(db=AT + 6 * MB + 1), dict(dx=AT), dict(dw=AT + MB),
    dict(dx=AT + 5 * MB), dict(db=AT + 3 * MB), dict(gated=1, ldz=11), dict(dx=AT + 7 * MB),
], ids=str)
def test_linear_backward_refusals(over):
    assert oz.load().ozaki2_linear_backward(*backward_args(**over)) == _lib.OZ2_E_INVALID


def test_backward_workspace():
    need = oz.ozaki2_linear_backward_workspace_bytes(oz.OZ2_F16, oz.OZ2_ACT_GELU, 0, 4, 6, 8)
    assert need >= 4 * 6 * 2
    L = oz.load()
    for over in (dict(ws=None), dict(wsb=need - 1), dict(ws=AT + 7 * MB + 128)):
        assert L.ozaki2_linear_backward(*backward_args(**over)) == _lib.OZ2_E_WORKSPACE
    assert oz.ozaki2_linear_backward_workspace_bytes(3, 0, 0, 4, 6, 8) == 0
    assert oz.ozaki2_linear_backward_workspace_bytes(0, 9, 0, 4, 6, 8) == 0
    # dZ of a gated layer: twice the outputs, in whole 64-byte pieces
    big = oz.ozaki2_linear_backward_workspace_bytes(oz.OZ2_BF16, oz.OZ2_ACT_SILU, 1, 1000, 2000, 8)
    assert big >= 1000 * 4000 * 2


def grouped_args(**over):
    a = dict(dtype=oz.OZ2_F32, act=0, gated=0, rows=9, groups=3, out=6, inp=8, off=AT + 8 * MB, x=AT,
             ldx=8, w=AT + MB, ldw=8, sw=48, bias=AT + 2 * MB, sb=6, y=AT + 3 * MB, ldy=6,
             z=AT + 4 * MB, ldz=6, ws=AT + 5 * MB, wsb=MB, stream=None)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over", [
    dict(groups=0), dict(groups=1025), dict(off=None), dict(off=AT + 8 * MB + 2), dict(sw=-1),
    dict(sb=-1), dict(x=None), dict(y=AT), dict(y=AT + MB + 4 * 96), dict(y=AT + 8 * MB - 8),
    dict(z=AT + 3 * MB + 4), dict(rows=-2), dict(ldy=5),
], ids=str)
def test_grouped_refusals(over):
    assert oz.load().ozaki2_grouped_linear(*grouped_args(**over)) == _lib.OZ2_E_INVALID


def test_grouped_backward_refusals():
    L = oz.load()
    base = dict(dtype=oz.OZ2_F32, act=0, gated=0, rows=9, groups=3, out=6, inp=8, off=AT + 8 * MB,
                dy=AT, lddy=6, x=AT + MB, ldx=8, w=AT + 2 * MB, ldw=8, sw=48, z=None, ldz=0,
                dx=AT + 3 * MB, lddx=8, dw=AT + 4 * MB, lddw=8, sdw=48, db=AT + 5 * MB, sdb=6,
                ws=AT + 6 * MB, wsb=MB, stream=None)
    for over in (dict(sdw=47), dict(sdb=5), dict(groups=0), dict(off=None), dict(dw=AT),
                 dict(act=1), dict(gated=1), dict(db=AT + 4 * MB)):
        assert L.ozaki2_grouped_linear_backward(*{**base, **over}.values()) == _lib.OZ2_E_INVALID, over
    assert L.ozaki2_grouped_linear_backward(*{**base, "ws": None}.values()) == _lib.OZ2_E_WORKSPACE


def test_workspace_apart_from_what_the_call_reads_and_writes():
    """the offsets of the groups, and all of the sort's arrays, are read or written
    while the workspace is"""
    L = oz.load()
    G, S, N, K = 3, 4096, 64, 65   # odd rows: copied into the workspace
    need = oz.ozaki2_grouped_linear_workspace_bytes(oz.OZ2_BF16, 0, S, G, N, K)
    assert need
    fwd = dict(dtype=oz.OZ2_BF16, act=0, gated=0, rows=S, groups=G, out=N, inp=K, off=AT + need - 16,
               x=AT + 64 * MB, ldx=K, w=AT + 128 * MB, ldw=K, sw=N * K, bias=None, sb=0,
               y=AT + 192 * MB, ldy=N, z=None, ldz=0, ws=AT, wsb=need, stream=None)
    assert L.ozaki2_grouped_linear(*fwd.values()) == _lib.OZ2_E_INVALID
    need = oz.ozaki2_grouped_linear_backward_workspace_bytes(oz.OZ2_BF16, 1, 0, S, G, N, K)
    bwd = dict(dtype=oz.OZ2_BF16, act=1, gated=0, rows=S, groups=G, out=N, inp=K, off=AT + need - 16,
               dy=AT + 64 * MB, lddy=N, x=AT + 80 * MB, ldx=K, w=AT + 128 * MB, ldw=K, sw=N * K,
               z=AT + 144 * MB, ldz=N, dx=AT + 192 * MB, lddx=K, dw=AT + 208 * MB, lddw=K, sdw=N * K,
               db=None, sdb=0, ws=AT, wsb=need, stream=None)
    assert L.ozaki2_grouped_linear_backward(*bwd.values()) == _lib.OZ2_E_INVALID
    need = oz.ozaki2_expert_sort_workspace_bytes(9000, 2, 4)
    sort = dict(T=9000, k=2, E=4, ids=AT, wide=1, ld=2, off=AT + MB, rows=AT + 2 * MB,
                slots=AT + 3 * MB, ws=AT + 4 * MB, wsb=need, s=None)
    for name in ("ids", "off", "rows", "slots"):
        over = {name: AT + 4 * MB + need - 8}
        assert L.ozaki2_expert_sort(*{**sort, **over}.values()) == _lib.OZ2_E_INVALID, name


def test_workspace_tensor_refusals():
    """the library sees a pointer and a number of bytes: these must be there"""
    from paper_2606_06510_amd import layers
    layers._init()
    cpu = torch.device("cpu")
    with pytest.raises(ValueError, match="contiguous"):
        layers._workspace(torch.zeros(1, dtype=torch.uint8).expand(1 << 20), 256, cpu)
    with pytest.raises(TypeError, match="workspace"):
        layers._workspace(b"0" * 512, 256, cpu)
    ws = torch.zeros(512, dtype=torch.uint8)
    assert layers._workspace(ws, 256, cpu)[1:] == (ws.data_ptr(), 512)


def test_expert_refusals():
    L = oz.load()
    bad = _lib.OZ2_E_INVALID
    sort = dict(T=9, k=2, E=4, ids=AT, wide=1, ld=2, off=AT + MB, rows=AT + 2 * MB, slots=AT + 3 * MB,
                ws=None, wsb=0, s=None)
    for over in (dict(T=-1), dict(k=0), dict(k=65), dict(E=0), dict(E=1025), dict(ids=None),
                 dict(ids=AT + 4), dict(ld=1), dict(off=None), dict(rows=None), dict(slots=None),
                 dict(rows=AT + MB + 4), dict(slots=AT + 8), dict(T=1 << 30)):
        assert L.ozaki2_expert_sort(*{**sort, **over}.values()) == bad, over
    need = oz.ozaki2_expert_sort_workspace_bytes(9000, 2, 4)
    assert need > 0
    big = {**sort, "T": 9000}
    assert L.ozaki2_expert_sort(*big.values()) == _lib.OZ2_E_WORKSPACE
    assert oz.ozaki2_expert_sort_workspace_bytes(9, 0, 4) == 0
    gather = dict(d=2, T=9, k=2, width=5, x=AT, ldx=5, slots=AT + MB, kept=AT + MB + 400, w=None,
                  xs=AT + 2 * MB, ldxs=5, s=None)
    for over in (dict(d=3), dict(T=-1), dict(k=0), dict(width=-1), dict(x=None), dict(ldx=4),
                 dict(slots=None), dict(kept=None), dict(xs=None), dict(ldxs=4), dict(xs=AT),
                 dict(xs=AT + MB), dict(x=AT + 1), dict(w=AT + 2 * MB + 4), dict(w=AT + MB + 1)):
        assert L.ozaki2_expert_gather(*{**gather, **over}.values()) == bad, over
    assert L.ozaki2_expert_gather(*{**gather, "T": 0}.values()) == 0
    comb = dict(d=1, T=9, k=2, width=5, ys=AT, ldys=5, slots=AT + MB, kept=AT + MB + 400, w=None,
                res=AT + 2 * MB, ldr=5, y=AT + 3 * MB, ldy=5, s=None)
    for over in (dict(ys=None), dict(ldys=4), dict(y=None), dict(y=AT), dict(res=AT + 3 * MB + 2),
                 dict(res=AT + 3 * MB, ldr=6), dict(slots=None), dict(y=AT + MB + 400)):
        assert L.ozaki2_expert_combine(*{**comb, **over}.values()) == bad, over
    back = dict(d=0, T=9, k=2, width=5, dy=AT, lddy=5, ys=AT + MB, ldys=5, slots=AT + 2 * MB,
                kept=AT + 2 * MB + 400, w=AT + 3 * MB, dys=AT + 4 * MB, lddys=5, dw=AT + 5 * MB, s=None)
    for over in (dict(dy=None), dict(ys=None), dict(w=None), dict(dys=AT), dict(dw=AT + MB),
                 dict(lddys=4), dict(dw=AT + 3 * MB), dict(dys=AT + 5 * MB), dict(slots=None)):
        assert L.ozaki2_expert_combine_backward(*{**back, **over}.values()) == bad, over


def test_nothing_to_do_is_no_error():
    L = oz.load()
    assert L.ozaki2_linear(*linear_args(rows=0, x=None, y=None)) == 0
    assert L.ozaki2_linear(*linear_args(out=0, w=None, y=None)) == 0
    assert L.ozaki2_linear_backward(*backward_args(dx=None, dw=None, db=None)) == 0
    assert L.ozaki2_linear_backward(*backward_args(rows=0, dw=None, db=None)) == 0


@pytest.fixture
def no_library_calls(monkeypatch):
    def boom(*a, **k):
        raise AssertionError("a library entry point was reached")
    for name in _lib.LAYER_EXPORTS:
        monkeypatch.setattr(_lib, name, boom)


def meta(*shape, dtype=torch.bfloat16):
    """A tensor that claims to be on the GPU is not to be had here; the checks of
    types, shapes and strides come before or beside that of the device."""
    return torch.zeros(shape, dtype=dtype)


def test_tensor_helpers_refuse(no_library_calls):
    x, w = meta(4, 8), meta(6, 8)
    with pytest.raises(ValueError, match="CUDA"):
        oz.linear(x, w)
    with pytest.raises(TypeError, match="torch tensor"):
        oz.linear([1.0], w)
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        oz.linear(x.double(), w)
    with pytest.raises(ValueError, match="activation"):
        oz.linear(x, w, activation="tanh")
    with pytest.raises(ValueError, match="int32 or int64"):
        oz.expert_sort(x, 4)
    with pytest.raises(ValueError, match="CUDA"):
        oz.expert_sort(torch.zeros((3, 2), dtype=torch.int64), 4)


def test_tensor_checks(no_library_calls, monkeypatch):
    from paper_2606_06510_amd import layers
    monkeypatch.setattr(layers, "_device", lambda name, t: t.device)
    x, w = meta(4, 8), meta(6, 8)
    for kw, match in [
            (dict(w=meta(6, 7)), "shape"), (dict(w=w.float()), "dtype"),
            (dict(w=meta(8, 6).t()), "adjacent"), (dict(x=meta(8, 4).t()), "adjacent"),
            (dict(x=meta(1, 8).expand(4, 8)), "overlap"), (dict(x=meta(8)), "dimensions"),
            (dict(bias=meta(5)), "shape"), (dict(bias=meta(12)[::2]), "adjacent"),
            (dict(residual=meta(4, 5)), "shape"), (dict(out=meta(3, 6)), "shape"),
            (dict(out=meta(4, 6).half()), "dtype"), (dict(w=meta(5, 8), gated=True), "even")]:
        with pytest.raises(ValueError, match=match):
            oz.linear(**{**dict(x=x, w=w), **kw})
    dy, z = meta(4, 6), meta(4, 6)
    for kw, match in [(dict(activation="silu"), "preactivation"), (dict(dy=meta(4, 5)), "shape"),
                      (dict(preactivation=meta(4, 5), activation="relu"), "shape"),
                      (dict(gated=True, preactivation=z), "shape"), (dict(dx=meta(4, 7)), "shape"),
                      (dict(dw=w.float()), "dtype"), (dict(dbias=meta(7)), "shape")]:
        with pytest.raises(ValueError, match=match):
            oz.linear_backward(**{**dict(dy=dy, x=x, w=w), **kw})
    w3, off = meta(3, 6, 8), torch.zeros(4, dtype=torch.int32)
    for kw, match in [(dict(w=w), "dimensions"), (dict(offsets=off.long()), "dtype"),
                      (dict(offsets=off[:3]), "shape"), (dict(bias=meta(3, 5)), "shape"),
                      (dict(offsets=torch.zeros(8, dtype=torch.int32)[::2]), "contiguous")]:
        with pytest.raises(ValueError, match=match):
            oz.grouped_linear(**{**dict(x=x, w=w3, offsets=off), **kw})
    slots = torch.zeros((4, 2), dtype=torch.int32)
    order = oz.ExpertOrder(off, torch.zeros(8, dtype=torch.int32), slots)
    with pytest.raises(ValueError, match="tokens"):
        oz.expert_gather(meta(5, 8), order)
    with pytest.raises(ValueError, match="dtype"):
        oz.expert_gather(x, order, weights=meta(4, 2))
    with pytest.raises(ValueError, match="shape"):
        oz.expert_combine(meta(7, 8), order)
    with pytest.raises(ValueError, match="shape"):
        oz.expert_combine_backward(x, meta(8, 8), order, torch.zeros((4, 3)))
    with pytest.raises(ValueError, match="dtype"):
        oz.expert_gather(x, order._replace(slots=slots.long()))
    for e in (0, 1025):
        with pytest.raises(ValueError, match="num_experts"):
            oz.expert_sort(torch.zeros((3, 2), dtype=torch.int64), e)


@pytest.mark.parametrize("act", lu.ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_plain_gradient_agrees_with_autograd(act, gated):
    g = torch.Generator().manual_seed(1)
    x, w, b = (torch.randn(s, generator=g, dtype=torch.float64).requires_grad_(True)
               for s in ((9, 5), (8, 5), (8,)))
    dy = torch.randn((9, 4 if gated else 8), generator=g, dtype=torch.float64)
    z = x @ w.t() + b
    y = lu.act(z[:, :4], act) * z[:, 4:] if gated else lu.act(z, act)
    want = torch.autograd.grad((y * dy).sum(), (x, w, b))
    got = lu.backward(dy, x, w, z, act, gated, torch.float32)
    for a, c in zip(got[:3], want):
        assert torch.allclose(a, c, rtol=1e-12, atol=1e-12)
