"""Plain 64-bit forms of the model operators on the CPU, and bounds on what the kernels'
32-bit arithmetic may differ from them (u, tiny and the types: layer_util).

A sum whose terms each pass through at most `depth` additions is off by at most depth
2^-24 of the sum of its terms' magnitudes; e^x in 32 bits by (2 + |x|) 2^-23 of itself
(the argument's rounding, times log2 e, and the function's own)."""
import math

import torch

from tests.layer_util import TINY, U, d, sum_error

E32 = 2.0 ** -24


# ----------------------------------------------------------------- router

def _sigmoid(l):
    return 1.0 / (1.0 + math.exp(-l)) if l >= 0 else math.exp(l) / (1.0 + math.exp(l))


def _first(values, n, allowed):
    """The n largest of `allowed`, of equal ones the lower index; NaN before all."""
    def key(i):
        v = values[i]
        return (0, 0.0, i) if math.isnan(v) else (1, -v, i)
    return sorted(allowed, key=key)[:n]


def route_row(l, bias, k, score, groups, top_groups, best, renorm, scale, chosen=None):
    """ids and weights of one token in Python's floats.  chosen: a function of the groups'
    values (None where a group is out) that gives the groups instead"""
    E = len(l)
    soft = score == "softmax"
    b = bias or [0.0] * E
    top = max((v for v in l if not math.isnan(v)), default=-math.inf)
    broken = soft and any(math.isnan(v) or v == math.inf for v in l)
    if soft:
        e = [0.0 if v == -math.inf or broken else math.exp(v - top) for v in l]
        total = sum(e)
        s = [math.nan if broken else (v / total if total else 0.0) for v in e]
    else:
        s = [math.nan if math.isnan(v) else (0.0 if v == -math.inf else 1.0 if v == math.inf
                                             else _sigmoid(v)) for v in l]
    scored = bias is not None or (groups > 1 and best > 1)
    c = [(s[i] + b[i]) if scored else l[i] for i in range(E)]
    inside = [i for i in range(E) if l[i] != -math.inf and b[i] != -math.inf]
    if groups > 1:
        per = E // groups
        value = []
        for g in range(groups):
            mine = [c[i] for i in inside if i // per == g]
            if any(math.isnan(v) for v in mine):
                value.append(math.nan)
            else:
                value.append(sum(sorted(mine, reverse=True)[:best]))
        some = [g for g in range(groups) if any(i // per == g for i in inside)]
        if chosen:
            kept = chosen([v if g in some else None for g, v in enumerate(value)])
        else:
            kept = _first(value, top_groups, some)
        inside = [i for i in inside if i // per in kept]
    ids = _first(c, k, inside)
    if soft and broken:
        w = [math.nan] * len(ids)
    elif not renorm:
        w = [s[i] for i in ids]
    elif soft:
        most = max((l[i] for i in ids), default=0.0)
        e = [math.exp(l[i] - most) for i in ids]
        w = [v / sum(e) for v in e]
    elif any(math.isnan(l[i]) for i in ids):
        w = [math.nan] * len(ids)
    else:
        # log sigmoid: scores that underflow keep their ratios
        q = [min(l[i], 0.0) - math.log1p(math.exp(-abs(l[i]))) for i in ids]
        e = [math.exp(v - max(q)) for v in q]
        w = [v / sum(e) for v in e]
    pad = k - len(ids)
    return ids + [-1] * pad, [scale * v for v in w] + [0.0] * pad


def route_weight_error(l, w):
    """Relative error of a weight: its exponential and those of the sum (at most as far from
    the largest logit as the row reaches), their sum, the division and the scale."""
    some = [v for v in l if math.isfinite(v)]
    reach = max(some) - min(some) if some else 0.0
    return abs(w) * (2 * (2 + reach + max(map(abs, some), default=0.0)) * 2.0 ** -23 + 40 * E32) + 2.0 ** -149


def route_backward(dw, l, ids, score, renorm, scale):
    """dlogits by differentiating the weights in 64 bits."""
    l = d(l).clone().requires_grad_(True)
    out = torch.zeros_like(l)
    dw, ids = d(dw), ids.cpu().long()
    for t in range(l.shape[0]):
        on = [j for j in range(ids.shape[1]) if 0 <= int(ids[t, j]) < l.shape[1]]
        if not on:
            continue
        at = ids[t, on]
        q = torch.log_softmax(l[t], 0) if score == "softmax" else torch.nn.functional.logsigmoid(l[t])
        q = q[at]
        p = torch.softmax(q, 0) if renorm else q.exp()
        g = torch.autograd.grad((scale * p * dw[t, on]).sum(), l)[0][t]
        out[t] = torch.where(torch.isneginf(l[t]), torch.zeros_like(g), g).detach()
    return out


def route_backward_error(dw, l, ids, scale):
    """Every term is at most max |g| of the row, relatively off as a weight is, a few dozen
    roundings beside."""
    l, dw = d(l), d(dw)
    fin = torch.where(torch.isfinite(l), l, torch.zeros_like(l))
    reach = (fin.amax(1) - fin.amin(1)) + fin.abs().amax(1)
    g = torch.where((ids.cpu() >= 0), dw.abs() * abs(scale), torch.zeros_like(dw)).amax(1)
    # the gradient is a difference of two terms of at most g each, for each choice
    return (g * (4 * (2 + reach) * 2.0 ** -23 + 160 * E32))[:, None].expand_as(l) * 2


# ------------------------------------------------------------------- norm

def depth(n):
    """Additions an entry of a row of n passes: its lane's (64 lanes at least), the lanes'"""
    return n / 64 + 24


def norm(x, w, b, eps):
    """y, stats and the bounds of their errors before rounding."""
    x, w, b = d(x), d(w), d(b)
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    c = x - mean
    var = (c * c).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    em = (depth(n) + 2) * E32 * x.abs().mean(1, keepdim=True)
    ec = em + E32 * c.abs()
    evar = (2 * c.abs() * ec + ec * ec).mean(1, keepdim=True) + (depth(n) + 4) * E32 * (var + eps + em * em)
    er = r * torch.minimum(evar / (var + eps) + 4 * E32, torch.ones_like(r) * 1e9)
    h, eh = c * r, ec * (r + er) + c.abs() * er + 2 * E32 * (c * r).abs()
    y, ey = (h, eh) if w is None else (h * w, eh * w.abs() + E32 * (h * w).abs())
    if b is not None:
        y, ey = y + b, ey + E32 * (y.abs() + b.abs())
    return y, torch.cat([mean, r], 1), ey, torch.cat([em, er], 1)


def norm_backward(dy, x, stats, w, res):
    """dx, dw, db and the bounds of their errors before rounding."""
    dy, x, stats, w, res = d(dy), d(x), d(stats), d(w), d(res)
    T, n = x.shape
    h = (x - stats[:, :1]) * stats[:, 1:]
    eh = 3 * E32 * h.abs()
    g = dy if w is None else dy * w
    eg = E32 * g.abs()
    r = stats[:, 1:].abs()
    mg, mh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    k = depth(n) + 3
    emg = (k * E32 * (g.abs() + eg) + eg).mean(1, keepdim=True)
    one = (g * h).abs() * 6 * E32
    emh = (k * E32 * ((g * h).abs() + one) + one).mean(1, keepdim=True)
    dx = stats[:, 1:] * (g - mg - h * mh)
    ex = r * (eg + emg + h.abs() * emh + eh * (mh.abs() + emh)
              + 4 * E32 * (g.abs() + mg.abs() + (h * mh).abs())) + 2 * E32 * dx.abs()
    if res is not None:
        dx, ex = dx + res, ex + E32 * (dx.abs() + res.abs())
    dw, db = (dy * h).sum(0), dy.sum(0)
    ew = sum_error(T) * (dy * h).abs().sum(0) + (dy.abs() * (eh + E32 * h.abs())).sum(0)
    eb = sum_error(T) * dy.abs().sum(0)
    return dx, dw, db, ex, ew, eb


# ------------------------------------------------------------------- loss

def _logits(x, w):
    x, w = d(x), d(w)
    return x @ w.t(), sum_error(x.shape[1]) * (x.abs() @ w.abs().t())


def loss(x, w, targets):
    """loss, lse and the bounds of their errors."""
    z, ez = _logits(x, w)
    T, V = z.shape
    t = targets.to(z.device).long()
    on = (t >= 0) & (t < V)
    if V == 0:
        lse = torch.full((T,), -math.inf, dtype=z.dtype, device=z.device)
        return torch.zeros_like(lse), lse, torch.zeros_like(lse), torch.zeros_like(lse)
    lse = torch.logsumexp(z, 1)
    top = z.amax(1)
    picked = z.gather(1, torch.where(on, t, 0)[:, None])[:, 0]
    p = torch.exp(z - lse[:, None])
    # the logits', the exponentials' (twice: those of chunks are joined), the sums' (8 of a lane,
    # the lanes', the chunks')
    far = (p * (2 + (top[:, None] - z))).sum(1) * 2.0 ** -23
    e = (p * ez).sum(1) + ez.amax(1) * 2.0 ** -20 + 3 * far + (V / 512 + 64) * E32 + 4 * E32
    elst = e + 2 * E32 * (lse.abs() + top.abs() + 1)
    eloss = e + ez.gather(1, torch.where(on, t, 0)[:, None])[:, 0] \
        + 2 * E32 * ((top - picked).abs() + (lse - top).abs() + 1)
    zero = torch.zeros_like(lse)
    return torch.where(on, lse - picked, zero), lse, torch.where(on, eloss, zero), elst


def loss_backward(dloss, x, w, targets, lse, dtype):
    """dx, dw and the bounds of their errors before the final rounding."""
    z, ez = _logits(x, w)
    x, w, g, lse = d(x), d(w), d(dloss), d(lse)
    T, V = z.shape
    t = targets.to(z.device).long()
    on = (t >= 0) & (t < V)
    g = torch.where(on, g, torch.zeros_like(g))[:, None]
    x = torch.where(on[:, None], x, torch.zeros_like(x))
    q = torch.exp(z - lse[:, None])
    q = torch.where(on[:, None], q, torch.zeros_like(q))
    hot = torch.zeros_like(q)
    hot[on.nonzero()[:, 0], t[on]] = 1.0
    dz = (q - hot) * g
    z = torch.where(on[:, None], z - lse[:, None], torch.zeros_like(z))
    e32 = (q * (torch.expm1(ez) + (2 + z.abs()) * 2.0 ** -23) + 3 * E32 * (q + hot)) * g.abs()
    e32 = torch.where(on[:, None], e32, torch.zeros_like(e32))
    # fp16 is scaled: the largest |dloss| is 2^14 at least
    tiny = TINY[dtype] if dtype != torch.float16 else TINY[dtype] * float(g.abs().max() if T else 0) / 2 ** 14
    # few tokens in 16 bits: what the first rounding leaves is kept, rounded in turn
    u = U[dtype] ** 2 if T <= 64 and dtype != torch.float32 else U[dtype]
    edz = e32 + u * (dz.abs() + e32) + tiny
    edz = torch.where(on[:, None], edz, torch.zeros_like(edz))
    m = dz.abs() + edz
    ex = edz @ w.abs() + sum_error(V) * (m @ w.abs())
    ew = edz.t() @ x.abs() + sum_error(T) * (m.t() @ x.abs())
    return dz @ w, dz.t() @ x, ex, ew
