"""Feed-forward layers of language models on the matrix cores (include/ozaki2/layers.h):
dense products with bias, activation and residual in the epilogue, tokens
in the order of their experts and back, the experts' products, and the gradients.

Argument checks and marshalling only; every step runs in the library's gfx950
kernels.  Matrices are row-major 2-D device tensors, one token per row: rows may
be any number of elements apart, the elements of a row are adjacent.  All of a
call's matrices have one dtype (float32, float16 or bfloat16) and one device.
Outputs and workspaces that are not given are allocated on the stream of the call
(``stream``, else torch's current one).

Autograd does not see these calls: a result requires no gradient, whatever the
inputs require, and nothing flows back through it by itself.  A training step calls the
gradients by name (each docstring says which), or wraps a function and its gradients in a
``torch.autograd.Function``.
"""
from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple

from . import _lib

ACTIVATIONS = {"none": _lib.OZ2_ACT_NONE, "relu": _lib.OZ2_ACT_RELU, "gelu": _lib.OZ2_ACT_GELU,
               "gelu_tanh": _lib.OZ2_ACT_GELU_TANH, "silu": _lib.OZ2_ACT_SILU}


class ExpertOrder(NamedTuple):
    """Token-expert pairs in the order of their experts (int32 device tensors).

    offsets [E + 1]: expert e has places offsets[e] .. offsets[e + 1] - 1, and
    offsets[E] pairs are kept; rows [tokens * top_k]: the pair (token * top_k +
    choice) at each place, dropped ones last; slots [tokens, top_k]: the place
    of each pair."""
    offsets: "torch.Tensor"   # noqa: F821
    rows: "torch.Tensor"      # noqa: F821
    slots: "torch.Tensor"     # noqa: F821


_torch = None
_raw_stream = None
_codes = {}

# bytes of workspace, functions of types and sizes alone
_linear_bytes = lru_cache(4096)(lambda *a: _lib.ozaki2_linear_workspace_bytes(*a))
_linear_backward_bytes = lru_cache(4096)(
    lambda *a: _lib.ozaki2_linear_backward_workspace_bytes(*a))
_grouped_bytes = lru_cache(4096)(lambda *a: _lib.ozaki2_grouped_linear_workspace_bytes(*a))
_grouped_backward_bytes = lru_cache(4096)(
    lambda *a: _lib.ozaki2_grouped_linear_backward_workspace_bytes(*a))
_sort_bytes = lru_cache(4096)(lambda *a: _lib.ozaki2_expert_sort_workspace_bytes(*a))


def _init():
    """torch is imported by the first call, as everywhere in this package"""
    global _torch, _raw_stream
    import torch
    # the handle alone, where torch offers it (a Stream object takes 2.5 us to make)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda index: torch.cuda.current_stream(index).cuda_stream)
    _codes.update({torch.float32: _lib.OZ2_F32, torch.float16: _lib.OZ2_F16,
                   torch.bfloat16: _lib.OZ2_BF16})
    _torch = torch


def _dtype(name, t):
    if _torch is None:
        _init()
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    code = _codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: expected float32, float16 or bfloat16, got {t.dtype}")
    return code


def _act(activation):
    try:
        return ACTIVATIONS[activation]
    except (KeyError, TypeError):
        raise ValueError(f"activation: expected one of {', '.join(ACTIVATIONS)}, "
                         f"got {activation!r}") from None


def _device(name, t):
    dev = t.device
    if dev.type != "cuda":
        raise ValueError(f"{name}: expected a tensor on a CUDA device, got one on {dev}")
    return dev


def _tensor(name, t, like, shape, dtype=None):
    """The C ABI sees pointers and sizes only: what does not match is refused here."""
    try:
        if (t.shape == shape and t.dtype is (dtype or like.dtype) and t.device == like.device
                and isinstance(t, _torch.Tensor)):
            return
    except AttributeError:
        pass
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not (dtype or like.dtype):
        raise ValueError(f"{name}: expected dtype {dtype or like.dtype}, got {t.dtype}")
    raise ValueError(f"{name}: expected a tensor on {like.device}, got one on {t.device}")


def _ld(name, t):
    """Distance of the rows of a tensor whose rows are contiguous (a dimension of
    size 1 carries no stride)."""
    if t.is_contiguous():
        return t.shape[-1] or 1
    rows, cols = t.shape[-2:]
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent (stride 1)")
    if rows <= 1:
        return max(cols, 1)
    ld = t.stride(-2)
    if ld < cols:
        raise ValueError(f"{name}: rows overlap (stride {ld} for rows of {cols})")
    return max(ld, 1)


def _matrix(name, t, like, shape):
    _tensor(name, t, like, shape)
    return _ld(name, t)


def _stack(name, t, like, shape):
    """Leading dimension and distance of the matrices of a 3-D tensor."""
    _tensor(name, t, like, shape)
    return _ld(name, t), t.stride(0) if shape[0] > 1 else 0


def _dense(name, t, like, shape, dtype):
    _tensor(name, t, like, shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")


def _vectors(name, t, like, shape):
    """Distance of the vectors (rows) of a 1-D or 2-D tensor."""
    _tensor(name, t, like, shape)
    if t.is_contiguous():
        return shape[-1]
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements must be adjacent (stride 1)")
    return t.stride(0) if len(shape) == 2 and shape[0] > 1 else 0


def _call(name, *args):
    """A library entry point with pointers and handles as integers already"""
    status = getattr(_lib.load(), name)(*args)
    if status:
        raise _lib.Ozaki2Error(name, status)


def _p(t):
    return None if t is None else t.data_ptr()


def _launch(device, stream, call):
    """call(stream handle) with ``device`` and the stream current, so that what
    it allocates belongs to the stream that uses it."""
    cuda = _torch.cuda
    if stream is None:
        if device.index == cuda.current_device():
            return call(_raw_stream(device.index))
        with cuda.device(device):
            return call(_raw_stream(device.index))
    if isinstance(stream, int):
        stream = (cuda.ExternalStream(stream, device=device) if stream
                  else cuda.default_stream(device))
    if stream.device != device:
        raise ValueError(f"stream: on {stream.device}, the tensors on {device}")
    with cuda.stream(stream):
        return call(stream.cuda_stream)


def _workspace(workspace, need, device):
    """(tensor, its pointer, its bytes)"""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = _torch.empty(need, dtype=_torch.uint8, device=device)
        return workspace, workspace.data_ptr(), need
    if not isinstance(workspace, _torch.Tensor):
        raise TypeError(f"workspace: expected a torch tensor, got {type(workspace).__name__}")
    if workspace.device != device:
        raise ValueError("workspace: on another device")
    if not workspace.is_contiguous():   # (its bytes would not all be there)
        raise ValueError("workspace: expected a contiguous tensor")
    # the library checks its size
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _dim2(name, t, n=2):
    try:
        if t.dim() == n:
            return t.shape
    except AttributeError:
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}") from None
    raise ValueError(f"{name}: expected {n} dimensions, got shape {tuple(t.shape)}")


# ------------------------------------------------------------------ dense

def linear(x, w, bias=None, residual=None, activation="none", gated=False,
           save_preactivation=False, out=None, workspace=None, stream=None):
    """f(x w^T + bias) + residual for x [T, in], w [out, in], bias [out] and
    residual [T, out]; f is ``activation``.

    gated: w has 2 out rows and bias 2 out entries, gates first, and the result
    is f(gates) * values + residual.  save_preactivation: returns (y, z) with z =
    x w^T + bias, rounded, as linear_backward takes it.  out may be residual
    itself.  Not recorded by autograd: its gradients are linear_backward's."""
    code, act, dev = _dtype("x", x), _act(activation), _device("x", x)
    T, K = _dim2("x", x)
    n2, _ = _dim2("w", w)
    if gated and n2 % 2:
        raise ValueError(f"w: a gated layer has an even number of rows, got {n2}")
    N = n2 // 2 if gated else n2
    ldx, ldw = _ld("x", x), _matrix("w", w, x, (n2, K))
    if bias is not None:
        _vectors("bias", bias, x, (n2,))
    ldr = _matrix("residual", residual, x, (T, N)) if residual is not None else 0
    ldy = _matrix("out", out, x, (T, N)) if out is not None else N
    need = _linear_bytes(code, gated, T, N, K)

    def call(s):
        y = x.new_empty((T, N)) if out is None else out
        z = x.new_empty((T, n2)) if save_preactivation else None
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_linear", code, act, gated, T, N, K, x.data_ptr(), ldx, w.data_ptr(), ldw,
              _p(bias), _p(residual), ldr, y.data_ptr(), ldy, _p(z), n2, ws, nb, s)
        return (y, z) if save_preactivation else y
    return _launch(dev, stream, call)


def linear_backward(dy, x, w, preactivation=None, activation="none", gated=False, need_dx=True,
                    need_dw=True, need_dbias=True, dx=None, dw=None, dbias=None, workspace=None,
                    stream=None):
    """(dx, dw, dbias) of ``linear`` from dy [T, out] and the pre-activation
    it saved (none without activation and gates); None for what is not needed.
    The residual's gradient is dy itself.  dx, dw, dbias: outputs to write into.

    The gradient at the pre-activation is rounded to the tensors' dtype before the
    products, as every operand of theirs: relatively 2^-9 in bfloat16; in float16 infinite
    beyond 65504.  float32 tensors keep it in 32 bits."""
    code, act, dev = _dtype("dy", dy), _act(activation), _device("dy", dy)
    T, N = _dim2("dy", dy)
    n2 = 2 * N if gated else N
    K = _dim2("x", x)[1]
    lddy, ldx, ldw = _ld("dy", dy), _matrix("x", x, dy, (T, K)), _matrix("w", w, dy, (n2, K))
    z, ldz = _preactivation(preactivation, act, gated, dy, (T, n2))
    for name, t, shape in (("dx", dx, (T, K)), ("dw", dw, (n2, K))):
        if t is not None:
            _matrix(name, t, dy, shape)
    if dbias is not None:
        _vectors("dbias", dbias, dy, (n2,))
    need = _linear_backward_bytes(code, act, gated, T, N, K)

    def call(s):
        gx = dy.new_empty((T, K)) if need_dx and dx is None else dx
        gw = dy.new_empty((n2, K)) if need_dw and dw is None else dw
        gb = dy.new_empty((n2,)) if need_dbias and dbias is None else dbias
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_linear_backward", code, act, gated, T, N, K, dy.data_ptr(), lddy,
              x.data_ptr(), ldx, w.data_ptr(), ldw, _p(z), ldz, _p(gx),
              _ld("dx", gx) if gx is not None else 0, _p(gw),
              _ld("dw", gw) if gw is not None else 0, _p(gb), ws, nb, s)
        return gx, gw, gb
    return _launch(dev, stream, call)


def _preactivation(z, act, gated, like, shape):
    if act == _lib.OZ2_ACT_NONE and not gated:
        return None, 0
    if z is None:
        raise ValueError("preactivation: needed for the slope of the activation "
                         "(save_preactivation of the forward call)")
    return z, _matrix("preactivation", z, like, shape)


# ---------------------------------------------------------------- experts

def _offsets(offsets, groups, like):
    _dense("offsets", offsets, like, (groups + 1,), _torch.int32)


def grouped_linear(x, w, offsets, bias=None, activation="none", gated=False,
                   save_preactivation=False, out=None, workspace=None, stream=None):
    """``linear`` of a group of layers: rows offsets[g] .. offsets[g + 1] - 1 of x
    [S, in] through w[g] ([G, out, in], gated 2 out) and bias[g].  offsets is an int32
    device tensor [G + 1]; the host never reads it.  Rows from offsets[G] on are zeros.
    Not recorded by autograd: its gradients are grouped_linear_backward's."""
    code, act, dev = _dtype("x", x), _act(activation), _device("x", x)
    S, K = _dim2("x", x)
    G, n2 = _dim2("w", w, 3)[:2]
    if gated and n2 % 2:
        raise ValueError(f"w: a gated layer has an even number of rows, got {n2}")
    N = n2 // 2 if gated else n2
    ldx = _ld("x", x)
    ldw, sw = _stack("w", w, x, (G, n2, K))
    _offsets(offsets, G, x)
    sb = _vectors("bias", bias, x, (G, n2)) if bias is not None else 0
    ldy = _matrix("out", out, x, (S, N)) if out is not None else N
    need = _grouped_bytes(code, gated, S, G, N, K)

    def call(s):
        y = x.new_empty((S, N)) if out is None else out
        z = x.new_empty((S, n2)) if save_preactivation else None
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_grouped_linear", code, act, gated, S, G, N, K, offsets.data_ptr(),
              x.data_ptr(), ldx, w.data_ptr(), ldw, sw, _p(bias), sb, y.data_ptr(), ldy, _p(z), n2,
              ws, nb, s)
        return (y, z) if save_preactivation else y
    return _launch(dev, stream, call)


def grouped_linear_backward(dy, x, w, offsets, preactivation=None, activation="none", gated=False,
                            need_dx=True, need_dw=True, need_dbias=True, dx=None, dw=None,
                            dbias=None, workspace=None, stream=None):
    """(dx, dw, dbias) of ``grouped_linear``: zeros in the rows from offsets[G] on
    and for groups without rows.  Rounding as in linear_backward."""
    code, act, dev = _dtype("dy", dy), _act(activation), _device("dy", dy)
    S, N = _dim2("dy", dy)
    n2 = 2 * N if gated else N
    K = _dim2("x", x)[1]
    G = _dim2("w", w, 3)[0]
    lddy, ldx = _ld("dy", dy), _matrix("x", x, dy, (S, K))
    ldw, sw = _stack("w", w, dy, (G, n2, K))
    _offsets(offsets, G, dy)
    z, ldz = _preactivation(preactivation, act, gated, dy, (S, n2))
    if dx is not None:
        _matrix("dx", dx, dy, (S, K))
    if dw is not None:
        _stack("dw", dw, dy, (G, n2, K))
    if dbias is not None:
        _vectors("dbias", dbias, dy, (G, n2))
    need = _grouped_backward_bytes(code, act, gated, S, G, N, K)

    def call(s):
        gx = dy.new_empty((S, K)) if need_dx and dx is None else dx
        gw = dy.new_empty((G, n2, K)) if need_dw and dw is None else dw
        gb = dy.new_empty((G, n2)) if need_dbias and dbias is None else dbias
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_grouped_linear_backward", code, act, gated, S, G, N, K, offsets.data_ptr(),
              dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw, sw, _p(z), ldz, _p(gx),
              _ld("dx", gx) if gx is not None else 0, _p(gw),
              _ld("dw", gw) if gw is not None else 0, gw.stride(0) if gw is not None else 0, _p(gb),
              gb.stride(0) if gb is not None else 0, ws, nb, s)
        return gx, gw, gb
    return _launch(dev, stream, call)


def expert_sort(experts, num_experts, workspace=None, stream=None):
    """The ExpertOrder of experts [tokens, top_k] (int32 or int64): stable; a
    value outside [0, num_experts) drops its pair."""
    if _torch is None:
        _init()
    torch = _torch
    if not isinstance(experts, torch.Tensor):
        raise TypeError(f"experts: expected a torch tensor, got {type(experts).__name__}")
    if experts.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"experts: expected int32 or int64, got {experts.dtype}")
    dev = _device("experts", experts)
    T, k = _dim2("experts", experts)
    ld = _ld("experts", experts)
    if num_experts < 1 or num_experts > _lib.OZ2_MAX_EXPERTS:
        raise ValueError(f"num_experts: expected 1 to {_lib.OZ2_MAX_EXPERTS}, got {num_experts}")
    need = _sort_bytes(T, k, num_experts)

    def call(s):
        kw = dict(dtype=torch.int32, device=dev)
        o = ExpertOrder(torch.empty(num_experts + 1, **kw), torch.empty(T * k, **kw),
                        torch.empty((T, k), **kw))
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_expert_sort", T, k, num_experts, experts.data_ptr(),
              experts.dtype is torch.int64, ld, o.offsets.data_ptr(), o.rows.data_ptr(),
              o.slots.data_ptr(), ws, nb, s)
        return o
    return _launch(dev, stream, call)


def _order(order, like, tokens=None):
    """(pointers to the slots and to the number of pairs kept, T, k)"""
    offsets, _, slots = order
    T, k = _dim2("order.slots", slots)
    if tokens is not None and T != tokens:
        raise ValueError(f"order.slots: expected {tokens} tokens, got {T}")
    _dense("order.slots", slots, like, (T, k), _torch.int32)
    n, = _dim2("order.offsets", offsets, 1)
    if n < 2:
        raise ValueError("order.offsets: expected at least 2 entries")
    _dense("order.offsets", offsets, like, (n,), _torch.int32)
    return slots.data_ptr(), offsets.data_ptr() + 4 * (n - 1), T, k


def _weights(weights, like, shape):
    _dense("weights", weights, like, shape, _torch.float32)
    return weights


def expert_gather(x, order, weights=None, out=None, stream=None):
    """x[t] at the places of its pairs: [tokens * top_k, width], zeros for dropped
    pairs; with weights (float32 [tokens, top_k]), times the pair's weight.  Not recorded
    by autograd.  The gradients from dxs: of x ``expert_combine(dxs, order, weights)``, of
    the weights ``expert_combine_backward(x, dxs, order, weights, need_dys=False)[1]``."""
    code, dev = _dtype("x", x), _device("x", x)
    T0, width = _dim2("x", x)
    slots, kept, T, k = _order(order, x, T0)
    ldx = _ld("x", x)
    if weights is not None:
        _weights(weights, x, (T, k))
    ldo = _matrix("out", out, x, (T * k, width)) if out is not None else max(width, 1)

    def call(s):
        xs = x.new_empty((T * k, width)) if out is None else out
        _call("ozaki2_expert_gather", code, T, k, width, x.data_ptr(), ldx, slots, kept,
              _p(weights), xs.data_ptr(), ldo, s)
        return xs
    return _launch(dev, stream, call)


def expert_combine(ys, order, weights=None, residual=None, out=None, stream=None):
    """residual[t] + the sum over a token's pairs of weight * ys[place]: [tokens,
    width].  Dropped pairs are left out.  It is the gradient of expert_gather with the same
    weights, or without.  out may be residual itself.  Not recorded by autograd: its
    gradients are expert_combine_backward's."""
    code, dev = _dtype("ys", ys), _device("ys", ys)
    S, width = _dim2("ys", ys)
    slots, kept, T, k = _order(order, ys)
    ldys = _matrix("ys", ys, ys, (T * k, width))
    if weights is not None:
        _weights(weights, ys, (T, k))
    ldr = _matrix("residual", residual, ys, (T, width)) if residual is not None else 0
    ldo = _matrix("out", out, ys, (T, width)) if out is not None else max(width, 1)

    def call(s):
        y = ys.new_empty((T, width)) if out is None else out
        _call("ozaki2_expert_combine", code, T, k, width, ys.data_ptr(), ldys, slots, kept,
              _p(weights), _p(residual), ldr, y.data_ptr(), ldo, s)
        return y
    return _launch(dev, stream, call)


def expert_combine_backward(dy, ys, order, weights, need_dys=True, need_dweights=True,
                            stream=None):
    """(dys, dweights) of ``expert_combine`` from dy [tokens, width]; zeros for
    dropped pairs, None for what is not needed.  The residual's gradient is dy."""
    code, dev = _dtype("dy", dy), _device("dy", dy)
    T0, width = _dim2("dy", dy)
    slots, kept, T, k = _order(order, dy, T0)
    lddy, ldys = _ld("dy", dy), _matrix("ys", ys, dy, (T * k, width))
    _weights(weights, dy, (T, k))

    def call(s):
        dys = dy.new_empty((T * k, width)) if need_dys else None
        dw = _torch.empty((T, k), dtype=_torch.float32, device=dev) if need_dweights else None
        _call("ozaki2_expert_combine_backward", code, T, k, width, dy.data_ptr(), lddy,
              ys.data_ptr(), ldys, slots, kept, weights.data_ptr(), _p(dys), max(width, 1), _p(dw),
              s)
        return dys, dw
    return _launch(dev, stream, call)
