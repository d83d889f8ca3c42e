"""The layer operators where arguments are at the edge of what they may be: offsets of
groups that do not ascend, infinities in the last row before an end, the most rows, parameters and
their gradients in one buffer."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device
from tests.test_gpu_layers import case, check_grouped, grouped_case, oz

pytestmark = pytest.mark.gpu

INF = float("inf")
GUARD = 4096   # bytes on either side of an output


def guarded(shape, dtype):
    """An output of the shape inside a buffer of bytes 0x5A, and the buffer"""
    n = torch.empty(0, dtype=dtype).element_size()
    for s in shape:
        n *= s
    buf = torch.full((n + 2 * GUARD,), 0x5A, dtype=torch.uint8, device=device())
    return buf[GUARD:GUARD + n].view(dtype).view(shape), buf


# rows, groups, in, out, gated: few rows a group, small and large tiles, copied operands
NOT_ASCENDING = [(300, 64, 200, 136, False), (700, 64, 200, 136, True), (2600, 5, 520, 4104, False),
                 (700, 64, 131, 137, False), (4096, 64, 64, 520, False)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S,G,K,N,gated", NOT_ASCENDING)
def test_offsets_that_do_not_ascend(S, G, K, N, gated, dtype):
    """no result is promised, but nothing beside the outputs and the workspace is
    written, and the next call is right"""
    m, dt = oz(), lu.DTYPES[dtype]
    off = [0] + [S * i // G for i in range(1, G)] + [S - 3]
    c = grouped_case(off, 3, K, N, dtype, gated, seed=91)
    n2 = 2 * N if gated else N
    code = {"bf16": m.OZ2_BF16, "fp32": m.OZ2_F32}[dtype]
    need = m.ozaki2_grouped_linear_backward_workspace_bytes(code, m.OZ2_ACT_SILU, gated, S, G, N, K)
    g = torch.Generator().manual_seed(92)
    for bad in ([0, S] * 600, [S, 0] * 600, [S - i for i in range(1200)], [-5, 2 ** 31 - 1, -2 ** 31] * 400,
                torch.randint(-S, 2 * S, (1200,), generator=g).tolist()):
        o = torch.tensor(bad[:G + 1], dtype=torch.int32, device=device())
        bufs = dict(y=guarded((S, N), dt), dx=guarded((S, K), dt), dw=guarded((G, n2, K), dt),
                    db=guarded((G, n2), dt), ws=guarded((need,), torch.uint8))
        m.grouped_linear(c["x"], c["w"], o, bias=c["b"], activation="silu", gated=gated,
                         out=bufs["y"][0])
        m.grouped_linear_backward(c["dy"], c["x"], c["w"], o, preactivation=c["z"], activation="silu",
                                  gated=gated, dx=bufs["dx"][0], dw=bufs["dw"][0],
                                  dbias=bufs["db"][0], workspace=bufs["ws"][0])
        torch.cuda.synchronize()
        for name, (_, buf) in bufs.items():
            assert bool((buf[:GUARD] == 0x5A).all()) and bool((buf[-GUARD:] == 0x5A).all()), name
    check_grouped(off, 3, c, "silu", gated)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("act", lu.ACTS)
def test_infinite_gate_in_the_last_row(act, dtype):
    """a gate that was stored as infinity makes its values' bias gradients infinite, with
    the sign of dY, whatever the number of rows is a multiple of"""
    N = 40
    for T in (1, 5, 8, 16, 17, 31, 33, 130):
        c = case(T, 24, N, dtype, True, seed=93)
        c["z"][T - 1, :N] = INF
        _, _, db = oz().linear_backward(c["dy"], c["x"], c["w"], preactivation=c["z"], activation=act,
                                        gated=True)
        assert torch.equal(db[N:], c["dy"][T - 1].sign() * INF), T
        assert bool(torch.isfinite(db[:N]).all()), T


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_infinite_gate_in_the_last_row_of_a_group(dtype):
    off, N = [0, 5, 5, 38, 54, 84, 85], 40
    for which in (0, 2, 4, 5):
        c = grouped_case(off, 3, 24, N, dtype, True, seed=94)
        last = off[which + 1] - 1
        c["z"][last, :N] = INF
        _, _, db = oz().grouped_linear_backward(c["dy"], c["x"], c["w"], c["off"], preactivation=c["z"],
                                                activation="silu", gated=True)
        assert torch.equal(db[which, N:], c["dy"][last].sign() * INF)
        db[which, N:] = 0.0
        assert bool(torch.isfinite(db).all())


def test_two_to_the_30_rows():
    """the most rows there may be: more workgroups than one dimension of a grid takes.
    All rows but 64 at the start, in the middle and at the end are zeros."""
    m, T, n = oz(), 1 << 30, 64
    c = case(3 * n, 8, 8, "bf16", False, seed=95)
    at = [0, T // 2 - n // 2, T - n]

    def spread(rows):
        t = torch.zeros((T, 8), dtype=torch.bfloat16, device=device())
        for i, a in enumerate(at):
            t[a:a + n] = rows[n * i:n * (i + 1)]
        return t

    def gathered(t):
        """the rows that are not zeros; the others are"""
        got = torch.cat([t[a:a + n] for a in at])
        for a in at:
            t[a:a + n] = 0
        assert not any(bool(part.any()) for part in t.split(T // 16))
        return got
    x = spread(c["x"])
    y, _, ey, _ = lu.forward(c["x"], c["w"], None, None, "none", False)
    lu.check(gathered(m.linear(x, c["w"])), y, ey, "y")
    dx, dw, db, ex, ew, eb = lu.backward(c["dy"], c["x"], c["w"], None, "none", False, torch.bfloat16)
    gx, gw, gb = m.linear_backward(spread(c["dy"]), x, c["w"])
    lu.check(gathered(gx), dx, ex, "dx")
    lu.check(gw, dw, ew, "dw")
    lu.check(gb, db, eb, "db")


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("off,K,N", [([0, 40, 40, 301, 330], 72, 56), ([0, 3, 9], 136, 33)])
def test_gradients_of_a_layer_in_one_buffer(off, K, N, dtype):
    """[layer][dW, dbias, one more entry], [layer][row][W, dW], [row][layer][dW]: the bits of the same call
    with outputs of their own, and nothing beside them"""
    m, dt, G = oz(), lu.DTYPES[dtype], len(off) - 1
    c = grouped_case(off, 0, K, N, dtype, False, seed=96)
    kw = dict(preactivation=c["z"], activation="gelu")
    dx, dw, db = m.grouped_linear_backward(c["dy"], c["x"], c["w"], c["off"], **kw)
    flat = torch.full((G, N * K + N + 1), 7.0, dtype=dt, device=device())
    gw, gb = flat[:, :N * K].view(G, N, K), flat[:, N * K:-1]
    got = m.grouped_linear_backward(c["dy"], c["x"], c["w"], c["off"], dw=gw, dbias=gb, **kw)
    assert torch.equal(got[0], dx) and torch.equal(gw, dw) and torch.equal(gb, db)
    assert bool((flat[:, -1] == 7).all())
    rows = torch.full((N, G, K), 7.0, dtype=dt, device=device()).transpose(0, 1)
    m.grouped_linear_backward(c["dy"], c["x"], c["w"], c["off"], dw=rows, need_dx=False, **kw)
    assert torch.equal(rows, dw)
    wide = torch.full((G, N, 2 * K), 7.0, dtype=dt, device=device())
    wide[..., :K] = c["w"]
    got = m.grouped_linear_backward(c["dy"], c["x"], wide[..., :K], c["off"], dw=wide[..., K:], **kw)
    assert torch.equal(wide[..., K:], dw) and torch.equal(wide[..., :K], c["w"])
    for e in range(G):   # (W's rows may be read another way, so dx is not bit for bit the same)
        r = slice(off[e], off[e + 1])
        gx, _, _, ex, _, _ = lu.backward(c["dy"][r], c["x"][r], c["w"][e], c["z"][r], "gelu", False, dt)
        lu.check(got[0][r], gx, ex, f"dx of {e}")
