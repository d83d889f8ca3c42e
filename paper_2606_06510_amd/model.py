"""What stands before and behind the layers of a language model
(include/ozaki2/model.h): the router that gives every token its experts and their weights,
layer norm, and the cross entropy over a vocabulary whose logits are not kept; and the
gradients.

As in ``layers``: argument checks and marshalling only; matrices are row-major 2-D device
tensors with adjacent elements in a row, of one dtype (float32, float16 or bfloat16) and on
one device; outputs and workspaces that are not given are allocated on the stream of the
call; autograd records none of these calls (each docstring names the gradient).
"""
from __future__ import annotations

import ctypes
import math
from functools import lru_cache

from . import _lib, layers
from .layers import (_call, _dense, _device, _dim2, _dtype, _launch, _ld, _matrix, _p, _workspace)

SCORES = {"softmax": _lib.OZ2_SCORE_SOFTMAX, "sigmoid": _lib.OZ2_SCORE_SIGMOID}

# bytes of workspace, functions of types and sizes alone
_norm_bytes = lru_cache(4096)(lambda *a: _lib.ozaki2_layer_norm_backward_workspace_bytes(*a))
_loss_bytes = lru_cache(4096)(lambda *a: _lib.ozaki2_linear_cross_entropy_workspace_bytes(*a))
_loss_backward_bytes = lru_cache(4096)(
    lambda *a: _lib.ozaki2_linear_cross_entropy_backward_workspace_bytes(*a))


def _score(score):
    try:
        return SCORES[score]
    except (KeyError, TypeError):
        raise ValueError(f"score: expected one of {', '.join(SCORES)}, got {score!r}") from None


def _range(name, value, lo, hi):
    if not lo <= value <= hi:
        raise ValueError(f"{name}: expected {lo} to {hi}, got {value}")


# A small call is mostly the host's.  Its plain form (dense tensors, nothing given to write
# into, the current device and stream) goes through the extension csrc/fastcall.cpp in one
# step, which answers None to every other; there, what holds for nearly every tensor is asked
# first and in few steps, and where it does not the checks that name the fault follow.

_fast = None


def _bind():
    """The extension, with the library's entry points (built beside the library, and as needed
    as it is)"""
    global _fast
    lib = _lib.load()
    if layers._torch is None:
        layers._init()
    try:
        from . import _fastcall
    except ImportError as e:
        raise RuntimeError(f"{_lib.HERE}/_fastcall.so is missing or cannot be loaded ({e}): build "
                           "it with __graft_entry__.build()") from e
    names = ("layer_norm", "layer_norm_backward", "layer_norm_backward_workspace_bytes",
             "expert_route", "expert_route_backward", "linear_cross_entropy",
             "linear_cross_entropy_workspace_bytes", "linear_cross_entropy_backward",
             "linear_cross_entropy_backward_workspace_bytes")
    _fastcall.bind(*(ctypes.cast(getattr(lib, "ozaki2_" + n), ctypes.c_void_p).value for n in names),
                   layers._raw_stream, layers._current_device)
    _fast = _fastcall
    return _fast


def _rows(name, t):
    """(type code, device, rows, columns, leading dimension) of a matrix"""
    try:
        T, K = t.shape
        code = layers._codes[t.dtype]
        if t.is_cuda and t.is_contiguous():
            return code, t.device, T, K, K or 1
    except (AttributeError, KeyError, TypeError, ValueError):
        pass
    return (_dtype(name, t), _device(name, t), *_dim2(name, t), _ld(name, t))


def _same(name, t, like, shape, dtype):
    """A contiguous tensor of this shape and type on the device of ``like``"""
    try:
        if (t.shape == shape and t.dtype is dtype and t.is_contiguous()
                and t.get_device() == like.get_device()):
            return
    except AttributeError:
        pass
    _dense(name, t, like, shape, dtype)


# ----------------------------------------------------------------- router

def _experts(logits):
    code, dev, T, E, ld = _rows("logits", logits)
    if E < 1 or E > _lib.OZ2_MAX_EXPERTS:
        raise ValueError(f"logits: expected 1 to {_lib.OZ2_MAX_EXPERTS} experts, got {E}")
    return code, dev, T, E, ld


def expert_route(logits, top_k, bias=None, score="softmax", groups=1, top_groups=1, group_best=2,
                 renormalize=True, scale=1.0, stream=None):
    """(ids, weights) of the ``top_k`` experts of every token from its logits [tokens,
    experts]: ids int32 [tokens, top_k], as expert_sort takes them, and weights float32
    [tokens, top_k], as expert_combine takes them.

    An expert's score s is the softmax over all experts or the sigmoid of its logit; the
    experts of largest s + bias are chosen, largest first, of equal ones the lower index
    (compared as in 64 bits; without a bias, unless groups are compared by sums of two, by the
    logits, also where scores round to the same number).  bias [experts], float32, decides the choice alone.
    groups > 1: the experts are so many equal ranges, a group's value is the sum of its
    group_best (1 or 2) largest s + bias, and only the top_groups largest groups are chosen
    from.  The weights are scale * s, with renormalize scale * s / (the sum of the chosen s).

    An expert whose logit or bias is -inf is out (and costs nothing, where a large finite bias
    makes the choice three times as slow).  Where fewer than top_k are left (all, in
    a row of padding), ids is -1, which drops the pair, and the weight 0.  NaN is larger than
    every number.  Not recorded by autograd: the gradient is expert_route_backward's."""
    kind = _score(score)
    if stream is None:
        done = (_fast or _bind()).expert_route(logits, top_k, bias, kind, groups, top_groups, group_best,
                                               renormalize, scale)
        if done is not None:
            return done
    code, dev, T, E, ld = _experts(logits)
    if groups != 1 or top_groups != 1:
        _range("groups", groups, 1, E)
        if E % groups:
            raise ValueError(f"groups: {E} experts are no {groups} equal groups")
        _range("top_groups", top_groups, 1, groups)
    if group_best not in (1, 2):
        raise ValueError(f"group_best: expected 1 or 2, got {group_best}")
    _range("top_k", top_k, 1, min(_lib.OZ2_MAX_TOPK, E // groups * top_groups))
    torch = layers._torch
    if bias is not None:
        _same("bias", bias, logits, (E,), torch.float32)

    def call(s):
        ids = torch.empty(T, top_k, dtype=torch.int32, device=dev)
        weights = torch.empty(T, top_k, dtype=torch.float32, device=dev)
        _call("ozaki2_expert_route", code, T, E, top_k, logits.data_ptr(), ld, _p(bias), kind, groups,
              top_groups, group_best, bool(renormalize), scale, ids.data_ptr(), weights.data_ptr(), s)
        return ids, weights
    return _launch(dev, stream, call)


def expert_route_backward(dweights, logits, ids, score="softmax", renormalize=True, scale=1.0,
                          dlogits=None, stream=None):
    """dlogits [tokens, experts], of the logits' dtype, from dweights (float32 [tokens,
    top_k], as expert_combine_backward gives them) and the ids that expert_route chose with the
    same score, renormalize and scale.  Choices of -1 take no part.  The bias has no
    gradient.  dlogits: an output to write into."""
    kind = _score(score)
    if stream is None and dlogits is None:
        done = (_fast or _bind()).expert_route_backward(dweights, logits, ids, kind, renormalize, scale)
        if done is not None:
            return done
    code, dev, T, E, ld = _experts(logits)
    T0, k = _dim2("ids", ids)
    if T0 != T:
        raise ValueError(f"ids: expected {T} tokens, got {T0}")
    _range("top_k", k, 1, min(_lib.OZ2_MAX_TOPK, E))
    torch = layers._torch
    _same("ids", ids, logits, (T, k), torch.int32)
    _same("dweights", dweights, logits, (T, k), torch.float32)
    ldd = _matrix("dlogits", dlogits, logits, (T, E)) if dlogits is not None else E

    def call(s):
        d = torch.empty(T, E, dtype=logits.dtype, device=dev) if dlogits is None else dlogits
        _call("ozaki2_expert_route_backward", code, T, E, k, dweights.data_ptr(), logits.data_ptr(),
              ld, ids.data_ptr(), kind, bool(renormalize), scale, d.data_ptr(), ldd, s)
        return d
    return _launch(dev, stream, call)


# ------------------------------------------------------------------- norm

def layer_norm(x, weight=None, bias=None, eps=1e-5, save_stats=False, out=None, stream=None):
    """(x - mean) / sqrt(variance + eps) * weight + bias for the rows of x [T, width];
    weight and bias [width].

    save_stats: returns (y, stats) with stats float32 [T, 2], each row's mean and 1 /
    sqrt(variance + eps), as layer_norm_backward takes them (NaN of rows of no width).  out may be x itself.  Not
    recorded by autograd: its gradients are layer_norm_backward's."""
    if stream is None and out is None:
        done = (_fast or _bind()).layer_norm(x, weight, bias, eps, bool(save_stats))
        if done is not None:
            return done
    code, dev, T, K, ldx = _rows("x", x)
    if not eps >= 0.0:
        raise ValueError(f"eps: expected a number of at least 0, got {eps}")
    if weight is not None:
        _same("weight", weight, x, (K,), x.dtype)
    if bias is not None:
        _same("bias", bias, x, (K,), x.dtype)
    ldy = _matrix("out", out, x, (T, K)) if out is not None else K or 1
    torch = layers._torch

    def call(s):
        y = torch.empty(T, K, dtype=x.dtype, device=dev) if out is None else out
        stats = torch.empty(T, 2, dtype=torch.float32, device=dev) if save_stats else None
        if save_stats and K == 0:
            stats.fill_(math.nan)   # 0 / 0: the library writes nothing where there is no width
        _call("ozaki2_layer_norm", code, T, K, x.data_ptr(), ldx, _p(weight), _p(bias), eps,
              y.data_ptr(), ldy, _p(stats), s)
        return (y, stats) if save_stats else y
    return _launch(dev, stream, call)


def layer_norm_backward(dy, x, stats, weight=None, residual=None, need_dx=True, need_dweight=True,
                        need_dbias=True, dx=None, dweight=None, dbias=None, workspace=None,
                        stream=None):
    """(dx, dweight, dbias) of ``layer_norm`` from dy [T, width] and the stats it saved;
    None for what is not needed.  residual [T, width], the gradient that flows past the norm, is
    added to dx (dx may be residual itself).  dx, dweight, dbias: outputs to write into."""
    if stream is None and workspace is None and dx is None and dweight is None and dbias is None:
        done = (_fast or _bind()).layer_norm_backward(dy, x, stats, weight, residual, need_dx,
                                                      need_dweight, need_dbias)
        if done is not None:
            return done
    code, dev, T, K, lddy = _rows("dy", dy)
    ldx = _matrix("x", x, dy, (T, K))
    _same("stats", stats, dy, (T, 2), layers._torch.float32)
    ldr = _matrix("residual", residual, dy, (T, K)) if residual is not None else 0
    if dx is not None:
        _matrix("dx", dx, dy, (T, K))
    for name, t in (("weight", weight), ("dweight", dweight), ("dbias", dbias)):
        if t is not None:
            _same(name, t, dy, (K,), dy.dtype)
    need = _norm_bytes(code, T, K) if need_dweight or need_dbias or dweight is not None \
        or dbias is not None else 0

    def call(s):
        gx = dy.new_empty((T, K)) if need_dx and dx is None else dx
        gw = dy.new_empty((K,)) if need_dweight and dweight is None else dweight
        gb = dy.new_empty((K,)) if need_dbias and dbias is None else dbias
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_layer_norm_backward", code, T, K, dy.data_ptr(), lddy, x.data_ptr(), ldx,
              stats.data_ptr(), _p(weight), _p(residual), ldr, _p(gx),
              _ld("dx", gx) if gx is not None else 0, _p(gw), _p(gb), ws, nb, s)
        return gx, gw, gb
    return _launch(dev, stream, call)


# ------------------------------------------------------------------- loss

def _targets(targets, like, T):
    try:
        if (targets.dtype is layers._torch.int64 and targets.shape == (T,) and targets.is_contiguous()
                and targets.get_device() == like.get_device()):
            return True
    except AttributeError:
        pass
    if not isinstance(targets, layers._torch.Tensor):
        raise TypeError(f"targets: expected a torch tensor, got {type(targets).__name__}")
    if targets.dtype not in (layers._torch.int32, layers._torch.int64):
        raise ValueError(f"targets: expected int32 or int64, got {targets.dtype}")
    _dense("targets", targets, like, (T,), targets.dtype)
    return targets.dtype is layers._torch.int64


def linear_cross_entropy(x, w, targets, workspace=None, stream=None):
    """(loss, lse) of tokens x [T, in] over a vocabulary w [vocab, in], float32 [T] each: with
    the logits z = x w^T, lse = log(sum(exp(z))) and loss = lse - z[target], 0 where the
    target (int32 or int64 [T]) is outside [0, vocab): a token that does not count.

    The logits are kept in 32 bits in the product's epilogue and never stored.  Not recorded
    by autograd: its gradients are linear_cross_entropy_backward's."""
    if stream is None and workspace is None:
        done = (_fast or _bind()).linear_cross_entropy(x, w, targets)
        if done is not None:
            return done
    code, dev, T, K, ldx = _rows("x", x)
    V, _ = _dim2("w", w)
    ldw = _matrix("w", w, x, (V, K))
    wide = _targets(targets, x, T)
    need = _loss_bytes(code, T, V, K)

    def call(s):
        out = x.new_empty((2, T), dtype=layers._torch.float32)
        loss, lse = out[0], out[1]
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_linear_cross_entropy", code, T, V, K, x.data_ptr(), ldx, w.data_ptr(), ldw,
              targets.data_ptr(), wide, loss.data_ptr(), lse.data_ptr(), ws, nb, s)
        return loss, lse
    return _launch(dev, stream, call)


def linear_cross_entropy_backward(dloss, x, w, targets, lse, need_dx=True, need_dw=True, dx=None,
                                  dw=None, workspace=None, stream=None):
    """(dx, dw) of ``linear_cross_entropy`` from dloss [T], float32 (of the mean over n
    tokens: 1 / n each), and the lse it returned; None for what is not needed.  Tokens that
    do not count have a zero row of dx and no part in dw, whatever their rows of x hold.  dx, dw:
    outputs to write into.

    The logits are computed again, a piece of the vocabulary at a time.  Their gradient is
    rounded to the tensors' dtype before the products, as every operand of theirs, in
    float16 times a power of two that keeps it in range (of up to 64 tokens in two parts,
    which hold twice the bits).  A caller that needs it in 32 bits for more tokens passes
    x.float() and w.float()."""
    if stream is None and workspace is None and dx is None and dw is None:
        done = (_fast or _bind()).linear_cross_entropy_backward(dloss, x, w, targets, lse, need_dx,
                                                                need_dw)
        if done is not None:
            return done
    code, dev, T, K, ldx = _rows("x", x)
    V, _ = _dim2("w", w)
    ldw = _matrix("w", w, x, (V, K))
    wide = _targets(targets, x, T)
    f32 = layers._torch.float32
    _same("dloss", dloss, x, (T,), f32)
    _same("lse", lse, x, (T,), f32)
    if dx is not None:
        _matrix("dx", dx, x, (T, K))
    if dw is not None:
        _matrix("dw", dw, x, (V, K))
    need = _loss_backward_bytes(code, T, V, K)

    def call(s):
        gx = x.new_empty((T, K)) if need_dx and dx is None else dx
        gw = x.new_empty((V, K)) if need_dw and dw is None else dw
        keep, ws, nb = _workspace(workspace, need, dev)
        _call("ozaki2_linear_cross_entropy_backward", code, T, V, K, dloss.data_ptr(), x.data_ptr(),
              ldx, w.data_ptr(), ldw, targets.data_ptr(), wide, lse.data_ptr(), _p(gx),
              _ld("dx", gx) if gx is not None else 0, _p(gw),
              _ld("dw", gw) if gw is not None else 0, ws, nb, s)
        return gx, gw
    return _launch(dev, stream, call)
