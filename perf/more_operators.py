"""What stands before and behind the feed-forward operators of a language model, and
how each is run: the router that gives every token its experts and their weights, layer
norm, and the cross entropy over a vocabulary whose logits are not kept; and the
gradients of all of them.

``listed()`` names the cases, ``draw()`` gives more of the same ranges.
``run()`` makes the calls a user's program makes where ``own`` is true, and
computes the same in elementary 32-bit torch operations where it is not (the
router's choice in 64 bits: neighbouring scores are closer than 32 bits tell);
``exact()`` is the definition in 64 bits.

Letters: T tokens (rows), K width, E experts, k choices per token, V vocabulary.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a few tokens being decoded find their experts: latency only
        dict(name="route_tokens", kind="route", dtype="bf16", T=8, E=64, k=8, score="softmax",
             bias=False, groups=1, top_groups=1, best=1, renorm=True, scale=1.0, pad=0.0, off=0),
        # a long batch over many experts in groups, balanced by a bias, from logits in 32
        # bits; some rows are padding
        dict(name="route_batch", kind="route", dtype="fp32", T=16384, E=256, k=8, score="sigmoid",
             bias=True, groups=8, top_groups=4, best=2, renorm=True, scale=2.5, pad=0.02, off=0),
        # the gradient of a plain softmax router in a training step
        dict(name="route_grad_batch", kind="route_grad", dtype="bf16", T=16384, E=128, k=8,
             score="softmax", bias=False, groups=1, top_groups=1, best=1, renorm=True, scale=1.0,
             pad=0.0, off=0),
        # scores that are not renormalised: every logit has a gradient; odd sizes, an
        # expert out of service
        dict(name="route_grad_odd", kind="route_grad", dtype="fp16", T=5000, E=27, k=3,
             score="softmax", bias=True, groups=1, top_groups=1, best=1, renorm=False, scale=1.0,
             pad=0.05, off=1),
        # the norm before a layer for one decoded token
        dict(name="norm_token", kind="norm", dtype="bf16", T=1, K=4096, bias=True, save=False),
        # the same for a training batch, keeping each row's statistics
        dict(name="norm_batch", kind="norm", dtype="bf16", T=16384, K=4096, bias=True, save=True),
        # its gradients, with the one that flows past the norm
        dict(name="norm_grad_batch", kind="norm_grad", dtype="bf16", T=16384, K=4096, bias=True,
             res=True),
        # gradients in full precision, odd sizes, rows unaligned
        dict(name="norm_grad_odd", kind="norm_grad", dtype="fp32", T=1500, K=1203, bias=True,
             res=False),
        # the score of a few tokens: W is read once
        dict(name="loss_tokens", kind="loss", dtype="bf16", T=4, K=4096, V=65536, ignore=0.0),
        # the loss of a long batch, the largest product
        dict(name="loss_batch", kind="loss", dtype="bf16", T=8192, K=4096, V=131072, ignore=0.05),
        # its gradients in a training step
        dict(name="loss_grad_batch", kind="loss_grad", dtype="bf16", T=4096, K=4096, V=65536,
             ignore=0.05, uneven=False),
        # a ragged batch over a vocabulary that is a multiple of nothing
        dict(name="loss_grad_odd", kind="loss_grad", dtype="fp16", T=777, K=1024, V=32003,
             ignore=0.3, uneven=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """As often a multiple of 64 as any number."""
    v = _log(rng, lo, hi)
    return max(64, 64 * (v // 64)) if rng.random() < 0.5 else v


def _cost(c):
    w = work(c)
    # 32-bit products cost some eight times as much
    return w["bytes"], w["flops"] * (8 if c["dtype"] == "fp32" and c["kind"].startswith("loss") else 1)


def draw(rng):
    most = [max(v) for v in zip(*(_cost(c) for c in listed()))]
    while True:
        c = _draw(rng)
        if all(a <= b for a, b in zip(_cost(c), most)):
            return c


def _draw(rng):
    kind = rng.choice(["route", "route_grad", "norm", "norm_grad", "loss", "loss_grad"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if kind in ("route", "route_grad"):
        c.update(T=_log(rng, 1, 20000), score=rng.choice(["softmax", "sigmoid"]),
                 bias=rng.random() < 0.5, groups=rng.choice([1, 1, 2, 4, 8]))
        c["E"] = c["groups"] * _log(rng, 4, 512 // c["groups"])
        c["top_groups"] = rng.randint(1, c["groups"])
        # groups are ranked by two experts' scores where a bias balances them
        c["best"] = 2 if c["bias"] and rng.random() < 0.7 else 1
        c.update(k=rng.randint(1, min(12, c["E"] // c["groups"] * c["top_groups"])),
                 renorm=rng.random() < 0.7, scale=rng.choice([1.0, 1.0, 2.5]),
                 pad=rng.choice([0.0, 0.0, 0.1]), off=rng.choice([0, 0, 1]))
    elif kind in ("norm", "norm_grad"):
        c.update(T=_log(rng, 1, 30000), K=_size(rng, 32, 16000), bias=rng.random() < 0.7)
        if kind == "norm":
            c.update(save=rng.random() < 0.7)
        else:
            c.update(res=rng.random() < 0.5)
    else:
        c.update(T=_log(rng, 1, 16384) if rng.random() < 0.8 else rng.randint(1, 64),
                 K=_size(rng, 64, 8192), V=_size(rng, 512, 131072),
                 ignore=rng.choice([0.0, 0.05, 0.5]))
        if kind == "loss_grad":
            c.update(uneven=rng.random() < 0.5)
    return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 31)


def _normal(gen, shape, dtype, scale=1.0, around=0.0):
    x = torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda")
    return x.mul_(scale).add_(around).to(dtype)


def prepare(case, seed):
    c, gen = case, _gen(seed)
    dt, T, kind = DTYPES[c["dtype"]], c["T"], c["kind"]
    s = dict(case=c)
    if kind in ("route", "route_grad"):
        # noisy logits around uneven popularities
        logits = torch.randn((T, c["E"]), generator=gen, device="cuda")
        logits += torch.randn((1, c["E"]), generator=gen, device="cuda").mul_(0.5)
        if c["off"]:
            logits[:, c["E"] // 2] = -math.inf
        if c["pad"]:
            pad = torch.rand((T, 1), generator=gen, device="cuda") < c["pad"]
            logits.masked_fill_(pad, -math.inf)
        s["logits"] = logits.to(dt)
        s["bias"] = (_normal(gen, (c["E"],), torch.float32, 0.05) if c["bias"] else None)
        if kind == "route_grad":
            s["ids"] = _plain_route(s["logits"], s["bias"], c)[0]
            s["dweights"] = _normal(gen, (T, c["k"]), torch.float32)
    elif kind in ("norm", "norm_grad"):
        # rows of unlike size, off their zero; one column stands out, as in a residual stream
        x = torch.randn((T, c["K"]), generator=gen, device="cuda")
        x *= torch.rand((T, 1), generator=gen, device="cuda").mul_(3.0).add_(0.3)
        x += torch.randn((T, 1), generator=gen, device="cuda").mul_(0.2)
        x[:, c["K"] // 3] += 8.0
        s["x"] = x.to(dt)
        del x
        s["weight"] = _normal(gen, (c["K"],), dt, 0.2, 1.0)
        s["bias"] = _normal(gen, (c["K"],), dt, 0.2) if c["bias"] else None
        if kind == "norm_grad":
            s["dy"] = _normal(gen, (T, c["K"]), dt)
            s["res"] = _normal(gen, (T, c["K"]), dt) if c["res"] else None
            s["stats"] = _plain_norm(s["x"], s["weight"], None)[1]
    else:
        K, V = c["K"], c["V"]
        s["x"] = _normal(gen, (T, K), dt)
        s["w"] = _normal(gen, (V, K), dt, 2.0 * K ** -0.5)
        # low indices are common
        u = torch.rand((T,), generator=gen, device="cuda", dtype=torch.float64)
        t = (V * u.pow(3)).long().clamp_(max=V - 1)
        if c["ignore"]:
            t.masked_fill_(torch.rand((T,), generator=gen, device="cuda") < c["ignore"], -100)
        s["targets"] = t
        if kind == "loss_grad":
            d = torch.full((T,), 1.0, device="cuda")
            if c["uneven"]:
                d.mul_(torch.rand((T,), generator=gen, device="cuda").add_(0.5))
            s["dloss"] = d.div_(T)
            rows = max(1, (1 << 28) // V)
            s["lse"] = torch.cat([_plain_loss(s["x"][r:r + rows], s["w"], t[r:r + rows])[1]
                                  for r in range(0, T, rows)])
    return s


# ------------------------------------------------------------- plain form

def _plain_route(logits, bias, c):
    T, E = logits.shape
    l = logits.double()
    out = l == -math.inf
    if c["score"] == "softmax":
        top = l.max(dim=1, keepdim=True)[0]
        e = torch.where(out, 0.0, torch.exp(l - top))
        s = e / e.sum(dim=1, keepdim=True)
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    v = s if bias is None else s + bias.double()
    v = torch.where(out, -math.inf, v)
    if c["groups"] > 1:
        per = E // c["groups"]
        best = torch.sort(v.reshape(T, c["groups"], per), dim=2, descending=True)[0][:, :, :c["best"]]
        some = best[:, :, 0] > -math.inf
        value = torch.where(best > -math.inf, best, 0.0).sum(dim=2)
        value = torch.where(some, value, -math.inf)
        order = torch.sort(value, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        keep = torch.zeros((T, c["groups"]), dtype=torch.bool, device=l.device)
        keep.scatter_(1, order, True)
        v = torch.where(keep.repeat_interleave(per, dim=1), v, -math.inf)
    v, ids = torch.sort(v, dim=1, descending=True, stable=True)
    v, ids = v[:, :c["k"]], ids[:, :c["k"]]
    there = v > -math.inf
    w = torch.where(there, s.gather(1, ids), 0.0)
    if c["renorm"]:
        w = torch.where(there, w / w.sum(dim=1, keepdim=True), 0.0)
    return torch.where(there, ids, -1).to(torch.int32), (c["scale"] * w).float()


def _plain_route_grad(dw, logits, ids, c):
    l = logits.float()
    there = ids >= 0
    at = ids.clamp(min=0).long()
    if c["score"] == "softmax":
        top = l.max(dim=1, keepdim=True)[0]
        e = torch.where(l == -math.inf, 0.0, torch.exp(l - top))
        s = e / e.sum(dim=1, keepdim=True)
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    mine = torch.where(there, s.gather(1, at), 0.0)
    g = torch.where(there, c["scale"] * dw, 0.0)
    if c["renorm"]:
        total = mine.sum(dim=1, keepdim=True)
        p = torch.where(there, mine / total, 0.0)
        g = (g - (p * g).sum(dim=1, keepdim=True)) / torch.where(total > 0, total, 1.0)
    ds = torch.zeros_like(l)
    ds.scatter_add_(1, at, torch.where(there, g, 0.0))
    if c["score"] == "softmax":
        s = torch.where(l == -math.inf, 0.0, s)
        return s * (ds - (s * ds).sum(dim=1, keepdim=True))
    return ds * s * (1.0 - s)


def _plain_norm(x, weight, bias):
    x = x.float()
    mean = x.mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(dim=1, keepdim=True) + 1e-5)
    y = (x - mean) * rstd * weight.float()
    if bias is not None:
        y = y + bias.float()
    return y, torch.cat([mean, rstd], dim=1)


def _plain_norm_grad(dy, x, stats, weight, res):
    mean, rstd = stats[:, :1], stats[:, 1:]
    dy = dy.float()
    h = (x.float() - mean) * rstd
    g = dy * weight.float()
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - h * (g * h).mean(dim=1, keepdim=True))
    if res is not None:
        dx = dx + res.float()
    return dx, (dy * h).sum(0), dy.sum(0)


def _plain_loss(x, w, targets):
    z = torch.matmul(x.float(), w.float().t())
    there = (targets >= 0) & (targets < w.shape[0])
    picked = z.gather(1, torch.where(there, targets, 0)[:, None])[:, 0]
    top = z.max(dim=1, keepdim=True)[0]
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))
    return torch.where(there, lse - picked, 0.0), lse


def _plain_loss_grad(dloss, x, w, targets, lse):
    x, w = x.float(), w.float()
    there = (targets >= 0) & (targets < w.shape[0])
    g = torch.where(there, dloss, 0.0)
    dz = torch.exp(torch.matmul(x, w.t()) - lse[:, None]) * g[:, None]
    dz.scatter_add_(1, torch.where(there, targets, 0)[:, None], -g[:, None])
    return torch.matmul(dz, w), torch.matmul(dz.t(), x)


def _plain(s):
    c = s["case"]
    dt, kind = DTYPES[c["dtype"]], c["kind"]
    if kind == "route":
        return list(_plain_route(s["logits"], s["bias"], c))
    if kind == "route_grad":
        return [_plain_route_grad(s["dweights"], s["logits"], s["ids"], c).to(dt)]
    if kind == "norm":
        y, stats = _plain_norm(s["x"], s["weight"], s["bias"])
        return [y.to(dt), stats] if c["save"] else [y.to(dt)]
    if kind == "norm_grad":
        dx, dw, db = _plain_norm_grad(s["dy"], s["x"], s["stats"], s["weight"], s["res"])
        return [dx.to(dt), dw.to(dt)] + ([db.to(dt)] if c["bias"] else [])
    if kind == "loss":
        return list(_plain_loss(s["x"], s["w"], s["targets"]))
    dx, dw = _plain_loss_grad(s["dloss"], s["x"], s["w"], s["targets"], s["lse"])
    return [dx.to(dt), dw.to(dt)]


# ------------------------------------------------- the library's operators

def _own(s):
    import paper_2606_06510_amd as oz
    c = s["case"]
    kind = c["kind"]
    if kind == "route":
        return list(oz.expert_route(s["logits"], c["k"], bias=s["bias"], score=c["score"],
                                    groups=c["groups"], top_groups=c["top_groups"],
                                    group_best=c["best"], renormalize=c["renorm"],
                                    scale=c["scale"]))
    if kind == "route_grad":
        return [oz.expert_route_backward(s["dweights"], s["logits"], s["ids"], score=c["score"],
                                         renormalize=c["renorm"], scale=c["scale"])]
    if kind == "norm":
        out = oz.layer_norm(s["x"], s["weight"], s["bias"], eps=1e-5, save_stats=c["save"])
        return list(out) if c["save"] else [out]
    if kind == "norm_grad":
        dx, dw, db = oz.layer_norm_backward(s["dy"], s["x"], s["stats"], weight=s["weight"],
                                            residual=s["res"], need_dbias=c["bias"])
        return [dx, dw] + ([db] if c["bias"] else [])
    if kind == "loss":
        return list(oz.linear_cross_entropy(s["x"], s["w"], s["targets"]))
    return list(oz.linear_cross_entropy_backward(s["dloss"], s["x"], s["w"], s["targets"],
                                                 s["lse"]))


def run(state):
    return _own(state) if own else _plain(state)


# -------------------------------------------------------------------- work

def work(case):
    """Each input read once and each output written once; the multiplications and
    additions of the products (the gradients of the loss: the logits again, which are
    not kept, and one product for each gradient), and a few operations an element
    elsewhere."""
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    T, kind = float(c["T"]), c["kind"]
    if kind == "route":
        return {"bytes": e * T * c["E"] + (4.0 * c["E"] if c["bias"] else 0.0) + 8.0 * T * c["k"],
                "flops": 4.0 * T * c["E"]}
    if kind == "route_grad":
        return {"bytes": 2.0 * e * T * c["E"] + 8.0 * T * c["k"], "flops": 8.0 * T * c["E"]}
    if kind == "norm":
        return {"bytes": e * (2 * T * c["K"] + c["K"] * (2 if c["bias"] else 1))
                + (8.0 * T if c["save"] else 0.0), "flops": 8.0 * T * c["K"]}
    if kind == "norm_grad":
        return {"bytes": e * (T * c["K"] * (4 if c["res"] else 3) + c["K"] * (3 if c["bias"] else 2))
                + 8.0 * T, "flops": 14.0 * T * c["K"]}
    K, V = c["K"], c["V"]
    if kind == "loss":
        return {"bytes": e * (T + V) * K + 16.0 * T, "flops": 2.0 * T * V * K}
    return {"bytes": 2.0 * e * (T + V) * K + 16.0 * T, "flops": 6.0 * T * V * K}


# ------------------------------------------------------------------- exact

_D = torch.float64


def _beaten(v):
    """How many of a row's values come before each: the larger ones, and equal ones of
    lower index."""
    n = torch.arange(v.shape[-1], device=v.device)
    a, b = v[..., :, None], v[..., None, :]
    return ((b > a) | ((b == a) & (n[None, :] < n[:, None]))).sum(-1)


def _exact_route(logits, bias, c):
    l = logits.to(_D)
    T, E = l.shape
    if c["score"] == "softmax":
        # (a row of padding is -inf throughout: no number)
        log_s = torch.log_softmax(l, dim=1)
    else:
        log_s = torch.nn.functional.logsigmoid(l)
    v = log_s.exp()
    if bias is not None:
        v = v + bias.to(_D)
    lost = -1e300    # below every score
    v = torch.where(torch.isneginf(l), lost, v)
    if c["groups"] > 1:
        g = v.reshape(T, c["groups"], -1)
        place = _beaten(g)
        value = (g * ((place < c["best"]) & (g > lost))).sum(2)
        value = torch.where((g > lost).any(2), value, lost)
        stays = (_beaten(value) < c["top_groups"]) & (value > lost)
        v = torch.where(stays[:, :, None], g, lost).reshape(T, E)
    place = torch.where(v > lost, _beaten(v), E)
    ids = torch.full((T, c["k"]), -1, dtype=torch.long, device=l.device)
    w = torch.full((T, c["k"]), -math.inf, dtype=_D, device=l.device)
    row, col = (place < c["k"]).nonzero(as_tuple=True)
    ids[row, place[row, col]] = col
    w[row, place[row, col]] = log_s[row, col]
    if c["renorm"]:
        w = torch.where(torch.isneginf(w), 0.0, torch.softmax(w, dim=1))
    else:
        w = w.exp()
    return ids, w * c["scale"]


def _exact_route_grad(dw, logits, ids, c):
    """By differentiating the weights as functions of the logits."""
    l = logits.to(_D)
    T = l.shape[0]
    grad = torch.zeros_like(l)
    live = (ids >= 0).any(1).nonzero()[:, 0]
    if live.numel() == 0:
        return grad
    with torch.enable_grad():
        z = l[live].requires_grad_(True)
        at = ids[live].long()
        off = at < 0
        log_s = (torch.log_softmax(z, dim=1) if c["score"] == "softmax"
                 else torch.nn.functional.logsigmoid(z))
        p = log_s.gather(1, at.clamp(min=0)).masked_fill(off, -math.inf)
        p = torch.softmax(p, dim=1) if c["renorm"] else p.exp()
        total = (c["scale"] * p * dw[live].to(_D)).masked_fill(off, 0.0).sum()
        g = torch.autograd.grad(total, z)[0]
    grad[live] = torch.where(torch.isneginf(l[live]), 0.0, g)
    return grad


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, T = c["kind"], c["T"]
    if kind == "route":
        rows = max(1, (1 << 27) // c["E"] ** 2)
        parts = [_exact_route(s["logits"][r:r + rows], s["bias"], c) for r in range(0, T, rows)]
        return [torch.cat(p) for p in zip(*parts)]
    if kind == "route_grad":
        return [_exact_route_grad(s["dweights"], s["logits"], s["ids"], c)]
    if kind == "norm":
        x = s["x"].to(_D)
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        r = (var + 1e-5).rsqrt()
        y = (x - mean).mul_(r).mul_(s["weight"].to(_D))
        if s["bias"] is not None:
            y += s["bias"].to(_D)
        return [y, torch.hstack([mean, r])] if c["save"] else [y]
    if kind == "norm_grad":
        # dx is what is left of dy weight rstd without its parts along ones and along h
        K = c["K"]
        m, r = s["stats"].to(_D).chunk(2, dim=1)
        h = s["x"].to(_D).sub_(m).mul_(r)
        dy = s["dy"].to(_D)
        out = [(dy * h).sum(dim=0)] + ([dy.sum(dim=0)] if c["bias"] else [])
        dy = dy.mul_(s["weight"].to(_D)).mul_(r)
        along = (dy * h).sum(dim=1, keepdim=True) / K
        dx = dy - dy.sum(dim=1, keepdim=True) / K - along * h
        if s["res"] is not None:
            dx += s["res"].to(_D)
        return [dx] + out
    x, w = s["x"].to(_D), s["w"].to(_D)
    rows = max(1, (1 << 28) // c["V"])
    if kind == "loss":
        loss, lse = [], []
        for r in range(0, T, rows):
            t = s["targets"][r:r + rows]
            z = x[r:r + rows] @ w.T
            l = torch.logsumexp(z, dim=1)
            n = torch.arange(t.numel(), device=t.device)
            loss.append(torch.where(t < 0, 0.0, l - z[n, t.clamp(min=0)]))
            lse.append(l)
        return [torch.cat(loss), torch.cat(lse)]
    dx, dw = torch.empty_like(x), torch.zeros_like(w)
    for r in range(0, T, rows):
        t = s["targets"][r:r + rows]
        d = (x[r:r + rows] @ w.T).sub_(s["lse"][r:r + rows, None]).exp_()
        n = (t >= 0).nonzero()[:, 0]
        d[n, t[n]] -= 1.0
        d *= torch.where(t >= 0, s["dloss"][r:r + rows].to(_D), 0.0)[:, None]
        dx[r:r + rows] = d @ w
        dw += d.T @ x[r:r + rows]
    return [dx, dw]
