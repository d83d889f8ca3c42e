"""The gradients as the docstrings name them: those of the weighted gather, and a layer's
operators inside torch.autograd functions."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device
from tests.test_gpu_experts import rows_case
from tests.test_gpu_layers import case, oz

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("T,k,E,width", [(1, 1, 1, 1), (9, 3, 8, 33), (64, 2, 8, 64), (33, 5, 6, 1130)])
def test_weighted_gather(T, k, E, width, dtype):
    m = oz()
    c, order, kept, slots = rows_case(T, k, E, width, dtype, seed=4)
    dxs = c["ys"]                                # any values; NaN for dropped pairs
    x, w = lu.d(c["x"]).requires_grad_(True), lu.d(c["w"]).requires_grad_(True)
    at = torch.tensor(slots).reshape(T, k)
    on = (at < kept).double()
    d = lu.d(dxs).clone()
    d[kept:] = 0.0
    terms = d[at.reshape(-1)].reshape(T, k, width)
    loss = ((w * on)[:, :, None] * x[:, None, :] * terms).sum()   # <gather, dxs>
    dx, dw = torch.autograd.grad(loss, (x, w))
    mag = ((w * on)[:, :, None] * terms).abs().sum(1).detach()
    lu.check(m.expert_combine(dxs, order, c["w"]), dx, lu.sum_error(k) * mag, "dx")
    got = m.expert_combine_backward(c["x"], dxs, order, c["w"], need_dys=False)
    assert got[0] is None
    lu.check(got[1], dw, lu.sum_error(width) * (x[:, None, :] * terms).abs().sum(2).detach(), "dweights")


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b):
        y, z = oz().linear(x, w, bias=b, activation="gelu", save_preactivation=True)
        ctx.save_for_backward(x, w, z)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, z = ctx.saved_tensors
        return oz().linear_backward(dy, x, w, preactivation=z, activation="gelu")


def test_inside_an_autograd_function():
    """called plainly a result requires no gradient; inside a Function the gradients
    are those called by name"""
    m, c = oz(), case(37, 44, 29, "fp32", False, seed=104)
    leaves = [c[n].contiguous().requires_grad_(True) for n in ("x", "w", "b")]
    plain = m.linear(*leaves, activation="gelu")
    assert not plain.requires_grad and plain.grad_fn is None
    y = Linear.apply(*leaves)
    assert y.requires_grad and torch.equal(y.detach(), plain)
    got = torch.autograd.grad((y * c["dy"]).sum(), leaves)
    _, z = m.linear(*leaves, activation="gelu", save_preactivation=True)
    want = m.linear_backward(c["dy"].contiguous(), leaves[0], leaves[1], preactivation=z, activation="gelu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(t.device == device() for t in got)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_precision_is_the_dtype_of_the_call(dtype):
    """the gradient at the pre-activation is an operand in the call's dtype: 16 bits round it
    once (lu.backward's bounds, which count that), the same values as float32 tensors do
    not"""
    m, c = oz(), case(150, 200, 88, dtype, False, seed=105)
    args = [c[n] for n in ("dy", "x", "w", "z")]
    for t in (args, [a.float() for a in args]):
        dx, dw, db, ex, ew, eb = lu.backward(*t, "silu", False, t[0].dtype)
        gx, gw, gb = m.linear_backward(t[0], t[1], t[2], preactivation=t[3], activation="silu")
        lu.check(gx, dx, ex, "dx")
        lu.check(gw, dw, ew, "dw")
        lu.check(gb, db, eb, "db")


def test_fp16_gradient_beyond_its_range():
    """dZ = 120000: infinite as an fp16 operand, 120000 in fp32"""
    m = oz()
    one = torch.ones((20, 8), dtype=torch.float16, device=device())
    args = [40000.0 * one[:, :4], one, 2.0 ** -6 * torch.cat([one, one])[:8], 3.0 * one]
    dx, _, _ = m.linear_backward(args[0], args[1], args[2], preactivation=args[3], activation="none",
                                 gated=True)
    assert bool(torch.isinf(dx).all())
    dx, _, _ = m.linear_backward(*(a.float() for a in args[:3]), preactivation=args[3].float(),
                                 activation="none", gated=True)
    assert bool((dx == 8 * 120000 / 64).all())
