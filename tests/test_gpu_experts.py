"""Tokens in the order of their experts and back: the sort, the gather, the
weighted sum and the gradients, against plain 64-bit forms."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device

pytestmark = pytest.mark.gpu


def oz():
    import paper_2606_06510_amd as m
    return m


def ids_of(T, k, E, seed, drop=0.0, wide=True, one=False):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, E, (T, k), generator=g)
    if one:
        ids[:] = E - 1
    ids[torch.rand((T, k), generator=g) < drop] = -1
    return (ids if wide else ids.to(torch.int32)).to(device())


SORTS = [(1, 1, 1, 0.0), (1, 2, 8, 0.0), (7, 3, 5, 0.5), (64, 1, 64, 0.0), (65, 2, 3, 0.1),
         (100, 8, 1024, 0.0), (1000, 4, 40, 0.05), (2048, 2, 16, 0.0), (2049, 2, 16, 0.0),
         (4097, 1, 7, 0.2), (3000, 6, 64, 0.02), (20000, 8, 128, 0.01), (30001, 1, 1000, 0.0),
         (50, 64, 33, 1.0)]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("T,k,E,drop", SORTS)
def test_sort(T, k, E, drop, wide):
    ids = ids_of(T, k, E, seed=T + k, drop=drop, wide=wide)
    o = oz().expert_sort(ids, E)
    offsets, rows, slots = lu.order(ids, E)
    assert o.offsets.tolist() == offsets
    assert o.rows.tolist() == rows
    assert o.slots.reshape(-1).tolist() == slots


def test_sort_values_outside_the_experts_and_strides():
    big = torch.full((300, 7), 99, device=device())
    big[:, :3] = ids_of(300, 3, 9, seed=1)
    big[::5, 1] = 9
    big[::7, 0] = -5
    big[3, 2] = 2 ** 40 + 1      # not 1: ids are compared in their own width
    ids = big[:, :3]
    o = oz().expert_sort(ids, 9)
    offsets, rows, slots = lu.order(ids, 9)
    assert o.offsets.tolist() == offsets and o.rows.tolist() == rows
    assert o.slots.reshape(-1).tolist() == slots
    o = oz().expert_sort(ids_of(5000, 2, 6, 2, one=True), 6)     # all to one expert
    assert o.offsets.tolist() == [0] * 6 + [10000] and o.rows.tolist() == list(range(10000))
    o = oz().expert_sort(ids[:0], 9)                             # no tokens
    assert o.offsets.tolist() == [0] * 10 and o.rows.numel() == 0


# tokens, choices, experts, width: one piece to many, odd widths
ROWS = [(1, 1, 1, 1), (3, 2, 4, 7), (5, 1, 2, 8), (9, 3, 8, 33), (64, 2, 8, 64), (33, 5, 6, 130),
        (200, 4, 16, 257), (17, 8, 9, 513), (70, 6, 12, 1024), (8, 2, 16, 4096), (31, 4, 4, 2001),
        (300, 9, 30, 65)]


def rows_case(T, k, E, width, dtype, drop=0.15, pad=0, shift=0, seed=0):
    from tests.test_gpu_layers import gen, rand
    g, dt = gen(100 + T + seed), lu.DTYPES[dtype]
    ids = ids_of(T, k, E, seed=T + width + seed, drop=drop)
    offsets, rows, slots = lu.order(ids, E)
    i32 = dict(dtype=torch.int32, device=device())
    order = oz().ExpertOrder(torch.tensor(offsets, **i32), torch.tensor(rows, **i32),
                             torch.tensor(slots, **i32).reshape(T, k))
    c = dict(x=rand(g, (T, width), dt, 1.0, pad, shift), ys=rand(g, (T * k, width), dt, 1.0, pad, shift),
             dy=rand(g, (T, width), dt, 1.0, pad, shift), r=rand(g, (T, width), dt, 1.0, pad, shift),
             w=torch.rand((T, k), generator=g).to(device()))
    c["ys"][offsets[-1]:] = float("nan")      # rows of dropped pairs are not read
    return c, order, offsets[-1], slots


def check_rows(c, order, kept, slots):
    m = oz()
    T, k = order.slots.shape
    dt = c["x"].dtype
    width = c["x"].shape[1]
    at = torch.tensor(slots).reshape(T, k)
    on = (at < kept).double()
    w = lu.d(c["w"])
    zero = torch.zeros((), dtype=torch.float64)
    # gather: a copy, or one product and one rounding
    xs = torch.zeros((T * k, width), dtype=torch.float64)
    xs[at.reshape(-1)] = (lu.d(c["x"])[:, None, :] * on[:, :, None]).reshape(T * k, width)
    assert torch.equal(lu.d(m.expert_gather(c["x"], order)), xs)
    ws = torch.zeros((T * k, 1), dtype=torch.float64)
    ws[at.reshape(-1)] = w.reshape(-1, 1)
    lu.check(m.expert_gather(c["x"], order, c["w"]), xs * ws, zero, "weighted gather")
    # combine
    ys = lu.d(c["ys"])
    ys[kept:] = 0.0
    terms = ys[at.reshape(-1)].reshape(T, k, width)
    for weights, res in [(True, True), (True, False), (False, True), (False, False)]:
        f = (w if weights else torch.ones_like(w))[:, :, None] * on[:, :, None]
        y, mag = (f * terms).sum(1), (f * terms).abs().sum(1)
        if res:
            y, mag = y + lu.d(c["r"]), mag + lu.d(c["r"]).abs()
        got = m.expert_combine(c["ys"], order, c["w"] if weights else None,
                               residual=c["r"] if res else None)
        lu.check(got, y, lu.sum_error(k) * mag, "combine")
    # its gradients
    dys, dw = m.expert_combine_backward(c["dy"], c["ys"], order, c["w"])
    dy = lu.d(c["dy"])
    want = torch.zeros((T * k, width), dtype=torch.float64)
    want[at.reshape(-1)] = ((w * on)[:, :, None] * dy[:, None, :]).reshape(T * k, width)
    lu.check(dys, want, zero, "dys")
    lu.check(dw, (terms * dy[:, None, :]).sum(2),
             lu.sum_error(width) * (terms * dy[:, None, :]).abs().sum(2), "dweights")
    only = m.expert_combine_backward(c["dy"], c["ys"], order, c["w"], need_dys=False)
    assert only[0] is None and torch.equal(only[1], dw)
    only = m.expert_combine_backward(c["dy"], c["ys"], order, c["w"], need_dweights=False)
    assert only[1] is None and torch.equal(only[0], dys)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,k,E,width", ROWS)
def test_rows(T, k, E, width, dtype):
    check_rows(*rows_case(T, k, E, width, dtype))


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("drop", [0.0, 1.0])
def test_rows_none_and_all_dropped(drop, dtype):
    """all dropped: tokens without any expert keep their residual, or are zero"""
    check_rows(*rows_case(50, 3, 5, 96, dtype, drop=drop))


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 3), (8, 8), (5, 1)])
def test_rows_strides(pad, shift, dtype):
    check_rows(*rows_case(40, 3, 5, 72, dtype, pad=pad, shift=shift))
    check_rows(*rows_case(6, 2, 5, 2000, dtype, pad=pad, shift=shift))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_offsets_past_32_bits(dtype):
    """rows so far apart that the last tokens' and places' begin past 2^32 bytes"""
    T, k, width = 150, 2, 40
    step = (1 << 24) // (2 if dtype == "bf16" else 4) + 8
    c, order, kept, slots = rows_case(T, k, 5, width, dtype)
    buf = torch.empty((T * k, step), dtype=lu.DTYPES[dtype], device=device())
    for name, at in (("x", 0), ("ys", 64), ("dy", 128), ("r", 192)):
        rows = c[name].shape[0]
        buf[:rows, at:at + width] = c[name]
        c[name] = buf[:rows, at:at + width]
    check_rows(c, order, kept, slots)
    ids = buf[:, 256:264].view(torch.int32)[:T, :k]
    ids.copy_(ids_of(T, k, 5, seed=7, drop=0.1, wide=False))
    o = oz().expert_sort(ids, 5)
    offsets, rows, slots = lu.order(ids, 5)
    assert o.offsets.tolist() == offsets and o.rows.tolist() == rows
    c, order, kept, slots = rows_case(T, k, 5, width, dtype, seed=3)
    xs = oz().expert_gather(c["x"], order, out=buf[:, :width])
    assert torch.equal(xs, oz().expert_gather(c["x"], order))


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_rows_outputs_given(dtype):
    """in place of the residual, and into column ranges of wider buffers"""
    m = oz()
    c, order, kept, slots = rows_case(60, 4, 7, 50, dtype)
    want = m.expert_combine(c["ys"], order, c["w"], residual=c["r"])
    buf = torch.full((60, 120), 5.0, dtype=c["x"].dtype, device=device())
    buf[:, 10:60] = c["r"]
    got = m.expert_combine(c["ys"], order, c["w"], residual=buf[:, 10:60], out=buf[:, 10:60])
    assert torch.equal(got, want) and bool((buf[:, :10] == 5).all()) and bool((buf[:, 60:] == 5).all())
    wide = torch.full((240, 99), 5.0, dtype=c["x"].dtype, device=device())
    got = m.expert_gather(c["x"], order, out=wide[:, 7:57])
    assert torch.equal(got, m.expert_gather(c["x"], order))
    assert bool((wide[:, :7] == 5).all()) and bool((wide[:, 57:] == 5).all())


def test_weights_of_the_gradient_against_differences():
    """<combine, dy> along a direction of the weights and of ys (linear in each: the
    difference of the 64-bit form is exact up to its rounding)"""
    c, order, kept, slots = rows_case(20, 3, 6, 40, "fp32", drop=0.2)
    dys, dw = oz().expert_combine_backward(c["dy"], c["ys"], order, c["w"])
    g = torch.Generator().manual_seed(3)
    at = torch.tensor(slots).reshape(20, 3)
    on = (at < kept).double()[:, :, None]
    ys, w, dy = lu.d(c["ys"]), lu.d(c["w"]), lu.d(c["dy"])
    ys[kept:] = 0.0

    def loss(ys, w):
        return float(((w[:, :, None] * on * ys[at.reshape(-1)].reshape(20, 3, 40)).sum(1) * dy).sum())
    vw, vy = torch.randn(w.shape, generator=g).double(), torch.randn(ys.shape, generator=g).double()
    for got, want, terms in [
            ((lu.d(dw) * vw).sum(), loss(ys, w + vw) - loss(ys, w), (lu.d(dw) * vw).abs().sum()),
            ((lu.d(dys) * vy).sum(), loss(ys + vy, w) - loss(ys, w), (lu.d(dys) * vy).abs().sum())]:
        assert abs(float(got) - want) < 1e-5 * float(terms)


def test_a_layer_of_experts_end_to_end():
    """sort, gather, two products, combine with the residual: the layer by its
    definition, token by token in 64 bits"""
    m, dev = oz(), device()
    T, k, E, H, F = 50, 2, 6, 64, 48
    g = torch.Generator().manual_seed(7)
    x = torch.randn((T, H), generator=g)
    w1, w2 = torch.randn((E, 2 * F, H), generator=g) * H ** -0.5, torch.randn((E, H, F), generator=g) * F ** -0.5
    ids = ids_of(T, k, E, seed=8, drop=0.1)
    w = torch.rand((T, k), generator=g)
    xd = x.to(dev)
    o = m.expert_sort(ids, E)
    h = m.grouped_linear(m.expert_gather(xd, o), w1.to(dev), o.offsets, activation="silu", gated=True)
    got = m.expert_combine(m.grouped_linear(h, w2.to(dev), o.offsets), o, w.to(dev), residual=xd)
    want = x.double().clone()
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            if e >= 0:
                z = w1[e].double() @ x[t].double()
                want[t] += w[t, j].double() * (w2[e].double() @ (lu.act(z[:F], "silu") * z[F:]))
    assert float((lu.d(got) - want).abs().max()) < 1e-4


def test_expert_graph_replays():
    m = oz()
    c, order, kept, slots = rows_case(100, 4, 8, 300, "bf16")
    ids = ids_of(3000, 2, 8, seed=5, drop=0.1)
    want = (list(m.expert_sort(ids, 8)) + [m.expert_gather(c["x"], order, c["w"])]
            + [m.expert_combine(c["ys"], order, c["w"], residual=c["r"])]
            + list(m.expert_combine_backward(c["dy"], c["ys"], order, c["w"])))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (list(m.expert_sort(ids, 8)) + [m.expert_gather(c["x"], order, c["w"])]
               + [m.expert_combine(c["ys"], order, c["w"], residual=c["r"])]
               + list(m.expert_combine_backward(c["dy"], c["ys"], order, c["w"])))
    for _ in range(4):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.randn(1000, device=device()).sum().item()
