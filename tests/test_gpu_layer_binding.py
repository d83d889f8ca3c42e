"""The entry points of include/ozaki2/layers.h through the binding of the same names, with
pointers, leading dimensions and workspaces passed by the caller: the bits of the tensor
functions."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device
from tests.test_gpu_layers import case, grouped_case, oz

pytestmark = pytest.mark.gpu

CODES = {"fp32": "OZ2_F32", "fp16": "OZ2_F16", "bf16": "OZ2_BF16"}


def empty(*shape, like=None, dtype=None):
    return torch.full(shape, 3, dtype=dtype or like.dtype, device=device())


def space(n):
    return torch.empty(n, dtype=torch.uint8, device=device()) if n else None


def streams():
    return [None, torch.cuda.current_stream(), torch.cuda.current_stream().cuda_stream]


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T", [3, 150])
def test_dense(T, dtype):
    m, K, N = oz(), 72, 45
    c, code, act = case(T, K, N, dtype, True, seed=101), getattr(m, CODES[dtype]), m.OZ2_ACT_SILU
    y, z = m.linear(c["x"], c["w"], bias=c["b"], residual=c["r"], activation="silu", gated=True,
                    save_preactivation=True)
    grads = m.linear_backward(c["dy"], c["x"], c["w"], preactivation=z, activation="silu", gated=True)
    for s in streams():
        gy, gz = empty(T, N, like=y), empty(T, 2 * N, like=y)
        need = m.ozaki2_linear_workspace_bytes(code, 1, T, N, K)
        ws = space(need)
        m.ozaki2_linear(code, act, 1, T, N, K, c["x"], K, c["w"], K, c["b"], c["r"], N, gy, N, gz, 2 * N,
                        ws, need, s)
        assert torch.equal(gy, y) and torch.equal(gz, z)
        dx, dw, db = empty(T, K, like=y), empty(2 * N, K, like=y), empty(2 * N, like=y)
        need = m.ozaki2_linear_backward_workspace_bytes(code, act, 1, T, N, K)
        ws = space(need)
        m.ozaki2_linear_backward(code, act, 1, T, N, K, c["dy"], N, c["x"], K, c["w"], K, z, 2 * N, dx, K,
                                 dw, K, db, ws, need, s)
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), grads))
    with pytest.raises(m.Ozaki2Error):
        m.ozaki2_linear(code, act, 1, T, N, K, c["x"], K - 1, c["w"], K, None, None, 0, gy, N, None, 0,
                        None, 0)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_grouped(dtype):
    m, off, K, N = oz(), [0, 9, 9, 150, 171], 72, 48
    c, code, act = grouped_case(off, 3, K, N, dtype, False, seed=102), getattr(m, CODES[dtype]), m.OZ2_ACT_GELU
    S, G = c["x"].shape[0], 4
    y, z = m.grouped_linear(c["x"], c["w"], c["off"], bias=c["b"], activation="gelu",
                            save_preactivation=True)
    grads = m.grouped_linear_backward(c["dy"], c["x"], c["w"], c["off"], preactivation=z, activation="gelu")
    gy, gz = empty(S, N, like=y), empty(S, N, like=y)
    need = m.ozaki2_grouped_linear_workspace_bytes(code, 0, S, G, N, K)
    ws = space(need)
    m.ozaki2_grouped_linear(code, act, 0, S, G, N, K, c["off"], c["x"], K, c["w"], K, N * K, c["b"], N, gy,
                            N, gz, N, ws, need)
    assert torch.equal(gy, y) and torch.equal(gz, z)
    dx, dw, db = empty(S, K, like=y), empty(G, N, K, like=y), empty(G, N, like=y)
    need = m.ozaki2_grouped_linear_backward_workspace_bytes(code, act, 0, S, G, N, K)
    ws = space(need)
    m.ozaki2_grouped_linear_backward(code, act, 0, S, G, N, K, c["off"], c["dy"], N, c["x"], K, c["w"], K,
                                     N * K, z, N, dx, K, dw, K, N * K, db, N, ws, need)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), grads))


@pytest.mark.parametrize("T", [40, 3000])
def test_experts(T):
    m, k, E, width = oz(), 3, 7, 50
    g = torch.Generator().manual_seed(103)
    ids = torch.randint(-1, E, (T, k), generator=g).to(device())
    order = m.expert_sort(ids, E)
    i32 = torch.int32
    o, rows, slots = empty(E + 1, dtype=i32), empty(T * k, dtype=i32), empty(T, k, dtype=i32)
    need = m.ozaki2_expert_sort_workspace_bytes(T, k, E)
    ws = space(need)
    m.ozaki2_expert_sort(T, k, E, ids, 1, k, o, rows, slots, ws, need)
    assert all(torch.equal(a, b) for a, b in zip((o, rows, slots), order))
    kept = o.data_ptr() + 4 * E
    x, r, dy = (torch.randn((T, width), generator=g).bfloat16().to(device()) for _ in range(3))
    w = torch.rand((T, k), generator=g).to(device())
    xs = empty(T * k, width, like=x)
    m.ozaki2_expert_gather(m.OZ2_BF16, T, k, width, x, width, slots, kept, w, xs, width)
    assert torch.equal(xs, m.expert_gather(x, order, w))
    y = empty(T, width, like=x)
    m.ozaki2_expert_combine(m.OZ2_BF16, T, k, width, xs, width, slots, kept, w, r, width, y, width)
    assert torch.equal(y, m.expert_combine(xs, order, w, residual=r))
    dys, dw = empty(T * k, width, like=x), empty(T, k, like=w)
    m.ozaki2_expert_combine_backward(m.OZ2_BF16, T, k, width, dy, width, xs, width, slots, kept, w, dys,
                                     width, dw)
    assert all(torch.equal(a, b) for a, b in zip((dys, dw), m.expert_combine_backward(dy, xs, order, w)))
