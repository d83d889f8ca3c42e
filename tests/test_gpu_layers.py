"""The dense and grouped products with their epilogues, and their gradients,
against plain 64-bit forms: types, activations, odd sizes and strides, empty and
uneven groups, rows outside the groups, streams and graphs."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device

pytestmark = pytest.mark.gpu

# rows, in, out: single tokens to several tiles, none a multiple of another
SIZES = [(1, 1, 1), (1, 64, 136), (1, 1000, 777), (2, 7, 13), (3, 4096, 40), (5, 136, 300),
         (16, 200, 64), (17, 33, 65), (31, 256, 128), (33, 512, 96), (64, 96, 64), (65, 8, 129),
         (100, 130, 200), (128, 128, 128), (129, 65, 127), (130, 320, 257), (200, 136, 300),
         (256, 256, 256), (257, 72, 264), (300, 1024, 520), (777, 99, 131)]


def oz():
    import paper_2606_06510_amd as m
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, shape, dtype, scale=1.0, pad=0, shift=0):
    """On the GPU; rows pad elements further apart, the first one shift elements in."""
    x = (torch.randn(shape, generator=g) * scale).to(dtype)
    wide = torch.full(shape[:-1] + (shape[-1] + pad,), float("nan"), dtype=dtype)
    flat = torch.full((wide.numel() + shift,), float("nan"), dtype=dtype, device=device())
    out = flat[shift:].view(wide.shape)[..., :shape[-1]]
    out.copy_(x)
    return out


def case(T, K, N, dtype, gated, seed, pad=0, shift=0):
    g, dt = gen(seed), lu.DTYPES[dtype]
    n2 = 2 * N if gated else N
    return dict(x=rand(g, (T, K), dt, 1.0, pad, shift),
                w=rand(g, (n2, K), dt, max(K, 1) ** -0.5, pad, shift),
                b=rand(g, (n2,), dt, 0.3, 0, shift), r=rand(g, (T, N), dt, 1.0, pad, shift),
                z=rand(g, (T, n2), dt, 1.5, pad, shift), dy=rand(g, (T, N), dt, 1.0, pad, shift))


def run_forward(c, act, gated, bias, res, save, **kw):
    y, z, ey, ez = lu.forward(c["x"], c["w"], c["b"] if bias else None, c["r"] if res else None,
                              act, gated)
    got = oz().linear(c["x"], c["w"], bias=c["b"] if bias else None,
                      residual=c["r"] if res else None, activation=act, gated=gated,
                      save_preactivation=save, **kw)
    if save:
        lu.check(got[1], z, ez, "z")
        got = got[0]
    lu.check(got, y, ey, "y")
    return got


def run_backward(c, act, gated, **kw):
    dt = c["x"].dtype
    dx, dw, db, ex, ew, eb = lu.backward(c["dy"], c["x"], c["w"], c["z"], act, gated, dt)
    gx, gw, gb = oz().linear_backward(c["dy"], c["x"], c["w"],
                                      preactivation=None if act == "none" and not gated else c["z"],
                                      activation=act, gated=gated, **kw)
    lu.check(gx, dx, ex, "dx")
    lu.check(gw, dw, ew, "dw")
    lu.check(gb, db, eb, "db")
    return gx, gw, gb


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_linear_sizes(size, dtype):
    T, K, N = size
    i = SIZES.index(size)
    for gated in (False, True):
        c = case(T, K, N, dtype, gated, seed=10 + i)
        run_forward(c, lu.ACTS[(i + gated) % 5], gated, bias=i % 2 == 0, res=i % 3 != 0,
                    save=i % 4 != 3)
        run_backward(c, lu.ACTS[(i + gated) % 5], gated)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", lu.ACTS)
def test_linear_activations(act, gated, dtype):
    for T in (4, 70):
        c = case(T, 96, 88, dtype, gated, seed=77)
        run_forward(c, act, gated, True, True, True)
        run_backward(c, act, gated)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (0, 1), (3, 5), (24, 8), (64, 3)])
@pytest.mark.parametrize("size", [(1, 264, 80), (40, 128, 72), (150, 272, 160), (300, 520, 264)])
def test_linear_strides(size, pad, shift, dtype):
    c = case(*size, dtype, False, seed=5, pad=pad, shift=shift)
    run_forward(c, "silu", False, True, True, True)
    run_backward(c, "silu", False)
    out = rand(gen(6), (size[0], size[2]), lu.DTYPES[dtype], 1.0, pad, shift)
    assert run_forward(c, "gelu", False, True, True, False, out=out) is out


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_linear_outputs_stay_inside_their_rows(dtype):
    """column slices of one buffer: what lies beside them keeps its values"""
    T, K, N = 130, 72, 45
    c = case(T, K, N, dtype, False, seed=8)
    buf = torch.full((T, 3 * N), 7.0, dtype=lu.DTYPES[dtype], device=device())
    buf[:, :N] = c["r"]
    c["r"] = buf[:, :N]
    run_forward(c, "relu", False, True, True, False, out=buf[:, N:2 * N])
    assert bool((buf[:, 2 * N:] == 7).all())
    want = buf[:, :N].clone()
    run_forward(c, "relu", False, True, True, False, out=buf[:, :N].copy_(want))   # in place
    assert bool((buf[:, 2 * N:] == 7).all())


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_linear_empty_sums(dtype):
    dt = lu.DTYPES[dtype]
    c = case(5, 1, 6, dtype, False, seed=3)
    x, w = c["x"][:, :0], c["w"][:, :0]
    got = oz().linear(x, w, bias=c["b"], residual=c["r"], activation="silu")
    want = lu.act(lu.d(c["b"]), "silu") + lu.d(c["r"])
    lu.check(got, want, lu.EACT * (1 + want.abs()))
    assert oz().linear(c["x"][:0], c["w"]).shape == (0, 6)
    assert oz().linear(c["x"], c["w"][:0]).shape == (5, 0)
    dx, dw, db = oz().linear_backward(c["dy"][:0], c["x"][:0], c["w"])   # no tokens
    assert dx.shape == (0, 1) and not dw.any() and not db.any() and dw.shape == (6, 1)
    dx, dw, db = oz().linear_backward(c["dy"][:, :0], c["x"], c["w"][:0])   # no outputs
    assert dx.shape == (5, 1) and not dx.any() and dw.shape == (0, 1)
    dx, dw, db = oz().linear_backward(c["dy"], x, w)   # no inputs
    assert dx.shape == (5, 0) and dw.shape == (6, 0)
    lu.check(db, lu.d(c["dy"]).sum(0), torch.full((6,), 1e-6, dtype=torch.float64))


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_linear_infinities_and_nan(dtype):
    """A NaN or infinity reaches the outputs that its row and column meet, and no
    others (nothing of a neighbouring row or a padded piece leaks in)."""
    for T, K, N in [(3, 40, 24), (70, 72, 56), (300, 264, 272)]:
        c = case(T, K, N, dtype, False, seed=4, pad=8)
        c["x"][1, K - 1] = float("nan")
        c["w"][2, 0] = float("inf")
        y = oz().linear(c["x"], c["w"], activation="none")
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[1] = True
        want[:, 2] = True
        assert torch.equal(bad, want)
        dy = c["dy"].clone()
        dy[0, N - 1] = float("nan")
        dx, dw, db = oz().linear_backward(dy, torch.nan_to_num(c["x"].contiguous()),
                                          torch.ones_like(c["w"]))
        assert bool(torch.isnan(dx[0]).all()) and bool(torch.isfinite(dx[1:]).all())
        assert bool(torch.isnan(dw[N - 1]).all()) and bool(torch.isfinite(dw[:-1]).all())
        assert bool(torch.isnan(db[-1])) and bool(torch.isfinite(db[:-1]).all())


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_linear_infinite_weights(dtype):
    """an infinite weight times positive inputs is an infinite output, in whichever part
    of the sum it lies: nothing beyond the sum's end meets it"""
    lines = {torch.float32: 32, torch.float16: 64, torch.bfloat16: 64}[lu.DTYPES[dtype]]
    for T in (1, 20, 70, 300):
        for K in (8, lines, 3 * lines, 9 * lines, 33 * lines + 8, 70 * lines):
            c = case(T, K, 24, dtype, False, seed=13)
            x = c["x"].abs() + 0.5
            for n, k in enumerate((0, K // 2, (K - 1) // lines * lines, K - 1)):
                c["w"][2 * n, k] = float("inf")
                c["w"][2 * n + 1, k] = -float("inf")
            for gated in (False, True):
                y = oz().linear(x, c["w"], gated=gated)
                z = torch.full((T, 24), float("inf"), device=device())
                z[:, 1::2] = -z[:, 1::2]
                if gated:   # gates 0 .. 7 are infinite, the values they meet finite
                    u = x.float() @ c["w"][12:].float().t()
                    assert torch.equal(y[:, :8].float(), (z[:, :8] * u[:, :8].sign()))
                else:
                    assert torch.equal(y[:, :8].float(), z[:, :8])
                assert bool(torch.isfinite(y[:, 8:]).all())


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_activations_at_large_arguments(act, dtype):
    """far out the functions are x or 0 and the slopes 1 or 0, without overflow
    on the way"""
    dt = lu.DTYPES[dtype]
    far = [150.0, 1e3, 6e4] + ([1e10, 1e25, 3e38] if dt != torch.float16 else [])
    x = torch.tensor([[v] for v in far] + [[-v] for v in far], dtype=dt, device=device())
    one = torch.ones((1, 1), dtype=dt, device=device())
    y = oz().linear(x, one, activation=act)
    n = len(far)
    assert torch.equal(y[:n], x[:n]) and not y[n:].any()
    dx, _, _ = oz().linear_backward(torch.ones_like(x), x, one, preactivation=x, activation=act)
    assert bool((dx[:n] == 1).all()) and not dx[n:].any()


def test_fp16_overflow_is_infinite():
    x = torch.full((20, 64), 60.0, dtype=torch.float16, device=device())
    y = oz().linear(x, x[:3])
    assert bool(torch.isinf(y).all())


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_linear_backward_wanted_gradients_alone(dtype):
    c = case(70, 48, 56, dtype, False, seed=12)
    full = run_backward(c, "gelu", False)
    for i, name in enumerate(("need_dx", "need_dw", "need_dbias")):
        need = dict.fromkeys(("need_dx", "need_dw", "need_dbias"), False)
        need[name] = True
        got = oz().linear_backward(c["dy"], c["x"], c["w"], preactivation=c["z"], activation="gelu",
                                   **need)
        for j in range(3):
            assert (got[j] is None) if j != i else torch.equal(got[j], full[j])


# one group of all, empty ones first, last and between, single rows, rows left over
GROUPS = [[0, 5], [0, 0, 3, 3, 40], [0, 1, 2, 130, 131], [0, 128, 256, 256], [0, 77, 77, 300],
          [0, 0, 0], [0] + [7 * i for i in range(1, 70)], [0, 33, 65, 97, 120, 120, 121]]


def grouped_case(off, left, K, N, dtype, gated, seed, pad=0, shift=0):
    S, G, g, dt = off[-1] + left, len(off) - 1, gen(seed), lu.DTYPES[dtype]
    n2 = 2 * N if gated else N
    c = dict(x=rand(g, (S, K), dt, 1.0, pad, shift),
             w=rand(g, (G, n2, K), dt, K ** -0.5, pad, shift),
             b=rand(g, (G, n2), dt, 0.3, pad, shift), z=rand(g, (S, n2), dt, 1.5, pad, shift),
             dy=rand(g, (S, N), dt, 1.0, pad, shift),
             off=torch.tensor(off, dtype=torch.int32, device=device()))
    for t in ("x", "z", "dy"):   # rows of no group are not read
        c[t][off[-1]:] = float("nan")
    return c


def check_grouped(off, left, c, act, gated, bias=True, save=True):
    got = oz().grouped_linear(c["x"], c["w"], c["off"], bias=c["b"] if bias else None,
                              activation=act, gated=gated, save_preactivation=save)
    y, z = got if save else (got, None)
    dx, dw, db = oz().grouped_linear_backward(
        c["dy"], c["x"], c["w"], c["off"],
        preactivation=None if act == "none" and not gated else c["z"], activation=act, gated=gated)
    n = off[-1]
    for t in (y, z, dx):
        assert t is None or not t[n:].any()
    for e in range(len(off) - 1):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            assert not dw[e].any() and not db[e].any()
            continue
        wy, wz, ey, ez = lu.forward(c["x"][r], c["w"][e], c["b"][e] if bias else None, None, act,
                                    gated)
        lu.check(y[r], wy, ey, f"y of {e}")
        if save:
            lu.check(z[r], wz, ez, f"z of {e}")
        gx, gw, gb, ex, ew, eb = lu.backward(c["dy"][r], c["x"][r], c["w"][e], c["z"][r], act, gated,
                                             c["x"].dtype)
        lu.check(dx[r], gx, ex, f"dx of {e}")
        lu.check(dw[e], gw, ew, f"dw of {e}")
        lu.check(db[e], gb, eb, f"db of {e}")


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("off", GROUPS, ids=[f"groups{i}" for i in range(len(GROUPS))])
def test_grouped_linear(off, dtype):
    i = GROUPS.index(off)
    for gated, (K, N), left in [(False, (64, 72), 0), (True, (40, 33), 5), (False, (136, 130), 140)]:
        c = grouped_case(off, left, K, N, dtype, gated, seed=20 + i)
        check_grouped(off, left, c, lu.ACTS[(i + gated) % 5], gated, bias=i % 2 == 0, save=i % 3 != 0)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_grouped_linear_strides(dtype):
    off = [0, 9, 9, 150, 171]
    c = grouped_case(off, 3, 72, 48, dtype, False, seed=31, pad=3, shift=1)
    check_grouped(off, 3, c, "gelu", False)
    c["w"] = c["w"][:1].expand(4, -1, -1)     # one set of weights for every group
    c["b"] = c["b"][:1].expand(4, -1)
    check_grouped(off, 3, c, "gelu", False)


def test_more_groups_than_a_wave():
    g = gen(9)
    sizes = torch.randint(0, 4, (1024,), generator=g).tolist()
    off = [0]
    for s in sizes:
        off.append(off[-1] + s)
    c = grouped_case(off, 2, 24, 16, "bf16", False, seed=32)
    y = oz().grouped_linear(c["x"], c["w"], c["off"], bias=c["b"])
    for e in [0, 1, 63, 64, 65, 500, 1022, 1023]:
        r = slice(off[e], off[e + 1])
        wy, _, ey, _ = lu.forward(c["x"][r], c["w"][e], c["b"][e], None, "none", False)
        lu.check(y[r], wy, ey, f"y of {e}")
    assert not y[off[-1]:].any()


@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("gelu_tanh", True)])
def test_gradients_against_differences(act, gated):
    """The change of <y, c> along a random direction, by central differences of the
    64-bit form, against the fp32 gradients.  Differences at h = 1e-4 leave h^2 / 6
    times a third derivative, some 1e-7 of the terms' size; the gradients' own sums
    are good to 50 x 2^-23."""
    T, K, N = 37, 44, 29
    c = case(T, K, N, "fp32", gated, seed=41)
    bias = c["b"]
    _, z = oz().linear(c["x"], c["w"], bias=bias, activation=act, gated=gated,
                       save_preactivation=True)
    dx, dw, db = oz().linear_backward(c["dy"], c["x"], c["w"], preactivation=z, activation=act,
                                      gated=gated)
    g, h = gen(42), 1e-4
    for name, grad in (("x", dx), ("w", dw), ("b", db)):
        v = torch.randn(c[name].shape, generator=g, dtype=torch.float64)

        def loss(s):
            t = {k: lu.d(c[k]) for k in ("x", "w", "b")}
            t[name] = t[name] + s * v
            return float((lu.forward(t["x"], t["w"], t["b"], None, act, gated)[0]
                          * lu.d(c["dy"])).sum())
        want = (loss(h) - loss(-h)) / (2 * h)
        got = float((lu.d(grad) * v).sum())
        scale = float((lu.d(grad) * v).abs().sum())
        assert abs(got - want) < 1e-5 * scale, (name, got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_same_bits_every_time(dtype):
    c = case(150, 700, 90, dtype, False, seed=51)
    first = run_backward(c, "silu", False) + (run_forward(c, "silu", False, True, True, False),)
    for _ in range(3):
        again = run_backward(c, "silu", False) + (run_forward(c, "silu", False, True, True, False),)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("T", [1, 40, 300])
def test_another_stream_and_graph(T):
    """on a stream of its own, and captured: every replay gives the eager bits"""
    c = case(T, 512, 264, "bf16", False, seed=61)
    eager = run_forward(c, "gelu", False, True, True, False)
    grads = run_backward(c, "gelu", False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = oz().linear(c["x"], c["w"], bias=c["b"], residual=c["r"], activation="gelu", stream=s)
    assert torch.cuda.current_stream() != s
    s.synchronize()
    assert torch.equal(y, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gy = oz().linear(c["x"], c["w"], bias=c["b"], residual=c["r"], activation="gelu")
        gg = oz().linear_backward(c["dy"], c["x"], c["w"], preactivation=c["z"], activation="gelu")
    for i in range(4):
        gy.zero_()
        for t in gg:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gy, eager) and all(torch.equal(a, b) for a, b in zip(gg, grads))
        torch.randn(1000, device=device()).sum().item()


def test_workspace_given():
    """a workspace of exactly the stated size, dirty, gives the same results"""
    m, dev = oz(), device()
    c = case(300, 520, 264, "bf16", True, seed=71)
    want = run_backward(c, "silu", True)
    need = m.ozaki2_linear_backward_workspace_bytes(m.OZ2_BF16, m.OZ2_ACT_SILU, 1, 300, 264, 520)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev)
    got = run_backward(c, "silu", True, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    if need > 256:
        with pytest.raises(m.Ozaki2Error):
            run_backward(c, "silu", True, workspace=ws[:need - 256])
