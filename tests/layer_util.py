"""Plain 64-bit forms of the layer operators on the CPU, and bounds on what the
kernels' arithmetic may differ from them.

Bounds.  u is the rounding of the type (bf16 2^-8, fp16 2^-11, fp32 2^-24); sums
of n products in 32 bits, whatever their order, are off by at most
(n + 4) 2^-23 of the sum of the products' magnitudes; an activation evaluated in
32 bits by at most (1 + |z|) 2^-20, and no activation here has a slope beyond
1.2 or a second derivative beyond 1."""
import math

import torch

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half the spacing of the numbers below the normal range
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
EACT = 2.0 ** -20


ON_GPU = False   # 64-bit references of large sizes: torch's fp64 on the GPU


def d(t):
    if t is None:
        return None
    return t.detach().double() if ON_GPU else t.detach().cpu().double()


def plan(dtype, side, M, N2, L, rows, groups=0, padded=False):
    """How the library runs a product: (few-row blocks, tile, splits, operands copied).
    side: 0 forward, 1 gradient of x, 2 of w."""
    import ctypes

    import paper_2606_06510_amd as oz
    f = oz.load().oz2_plan_of
    ll, i = ctypes.c_longlong, ctypes.c_int
    f.argtypes, f.restype = [i, i, ll, ll, ll, i, i, i, ctypes.POINTER(i)], None
    out = (i * 4)()
    f({"fp32": 0, "fp16": 1, "bf16": 2}[dtype], side, M, N2, L, rows, groups, padded, out)
    return tuple(out)


def plans(T, K, N, dtype, gated, sloped, groups=0):
    """The three products of a layer"""
    n2 = 2 * N if gated else N
    return (plan(dtype, 0, T, n2, K, T, groups), plan(dtype, 1, T, K, n2, T, groups, sloped),
            plan(dtype, 2, n2, K, T, T, groups, sloped))


def act(z, name):
    if name == "none":
        return z.clone()
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z)


def slope(z, name):
    """By differentiating act, not by a second formula."""
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act(z, name).sum(), z)[0]


def sum_error(n):
    return (n + 4) * 2.0 ** -23


def forward(x, w, bias, res, name, gated):
    """y, z and the bounds of their errors before the final rounding."""
    x, w, bias, res = d(x), d(w), d(bias), d(res)
    z = x @ w.t()
    mag = x.abs() @ w.abs().t()
    if bias is not None:
        z, mag = z + bias, mag + bias.abs()
    ez = sum_error(x.shape[1]) * mag
    if gated:
        n = z.shape[1] // 2
        a, u, ea, eu = z[:, :n], z[:, n:], ez[:, :n], ez[:, n:]
        f = act(a, name)
        ef = 1.2 * ea + EACT * (1 + a.abs())
        y, ey = f * u, ef * u.abs() + (f.abs() + ef) * eu + 2.0 ** -23 * (f * u).abs()
    else:
        y, ey = act(z, name), 1.2 * ez + EACT * (1 + z.abs()) * (name != "none")
    if res is not None:
        y, ey = y + res, ey + 2.0 ** -23 * (y.abs() + res.abs())
    return y, z, ey, ez


def backward(dy, x, w, z, name, gated, dtype):
    """dx, dw, db and the bounds of their errors before the final rounding."""
    u = U[dtype]
    dy, x, w, z = d(dy), d(x), d(w), d(z)
    if gated:
        n = dy.shape[1]
        a, v = z[:, :n], z[:, n:]
        dz = torch.cat([dy * v * slope(a, name), dy * act(a, name)], 1)
        e32 = torch.cat([(dy * v).abs(), dy.abs()], 1) * torch.cat([1 + a.abs()] * 2, 1) * 4 * EACT
    elif name != "none":
        dz = dy * slope(z, name)
        e32 = dy.abs() * (1 + z.abs()) * 4 * EACT
    else:
        dz, e32 = dy, torch.zeros_like(dy)
    edz = e32 + (u * (dz.abs() + e32) + TINY[dtype] if name != "none" or gated else 0.0)
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    m = dz.abs() + edz
    ex = edz @ w.abs() + sum_error(dz.shape[1]) * (m @ w.abs())
    ew = edz.t() @ x.abs() + sum_error(dz.shape[0]) * (m.t() @ x.abs())
    eb = e32.sum(0) + sum_error(dz.shape[0]) * m.sum(0)
    return dx, dw, db, ex, ew, eb


def check(got, want, err, what=""):
    """|got - want| within the bound and one rounding to got's type."""
    u, tiny = U[got.dtype], TINY[got.dtype]
    g = d(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    tol = err + u * (want.abs() + err) + tiny
    bad = ~((g - want).abs() <= tol)
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: "
                             f"{float(g[at])} for {float(want[at])}, bound {float(tol[at])}")


def order(experts, E):
    """offsets, rows, slots by the definition, in Python integers."""
    flat = experts.cpu().reshape(-1).tolist()
    keyed = sorted(range(len(flat)), key=lambda p: (flat[p] if 0 <= flat[p] < E else E, p))
    slots = [0] * len(flat)
    for place, p in enumerate(keyed):
        slots[p] = place
    offsets = [sum(1 for v in flat if 0 <= v < e) for e in range(E + 1)]
    return offsets, keyed, slots
