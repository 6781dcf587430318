"""Plain 64-bit forms of layer norm, routing, the experts' rows and the softmax loss, and how far an implementation with fp32 arithmetic may
be from them.

Tolerances.  u = 2^-24.  A sum whose longest chain of additions has D links is off by at most D u sum |terms|; what is known of the
kernels' chains is said at each sum.  Errors of inputs of a step are carried through it to first order.  Results are rounded
to their type by half a step, eps / 2 of the value, plus half of the smallest number below the normal range (`rounding`).
"""
import math

import torch

from dense_ref import U, check, rounding  # noqa: F401


# ---- layer norm
def norm64(x, weight=None, bias=None, eps=1e-5, grad=None):
    """out with its tolerance and, with `grad`, (dx, dweight, dbias) with theirs: dictionaries of pairs."""
    dtype, n, rows = x.dtype, x.shape[1], x.shape[0]
    x = x.double()
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(n, dtype=torch.float64) if bias is None else bias.double()
    D = 64 + n // 256  # a thread adds at most 32 elements of a row that fits the registers, n / 512 of another; then at most 9 + 8 joins
    mean = x.mean(1, keepdim=True)
    d = x - mean
    em = D * U * x.abs().mean(1, keepdim=True) + 2 * U * mean.abs()
    ed = em + U * d.abs()
    var = (d * d).mean(1, keepdim=True)
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (D + 4) * U * var
    rstd = 1 / (var + eps).sqrt()
    rel = 0.55 * ev / (var + eps) + 6 * U
    xh = d * rstd
    eh = xh.abs() * rel + ed * rstd + 2 * U * xh.abs()
    y = xh * w + b
    out = dict(out=(y, w.abs() * eh + 2 * U * ((xh * w).abs() + b.abs()) + rounding(y, dtype)))
    if grad is None:
        return out
    g = grad.double()
    h = g * w
    s, sx = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    es = (D + 4) * U * h.abs().mean(1, keepdim=True)
    esx = (h.abs() * eh).mean(1, keepdim=True) + (D + 4) * U * (h * xh).abs().mean(1, keepdim=True)
    dx = rstd * (h - s - xh * sx)
    size = h.abs() + s.abs() + (xh * sx).abs()
    out["dx"] = (dx, rstd * (es + xh.abs() * esx + eh * sx.abs() + 6 * U * size) + rel * rstd * size + rounding(dx, dtype))
    R = 100 + rows // 64  # links over the rows: at least 64 workgroups share them, 16 rows each are joined, then 48 more
    dw, db = (g * xh).sum(0), g.sum(0)
    out["dweight"] = (dw, (g.abs() * eh).sum(0) + (R + 2) * U * (g * xh).abs().sum(0) + rounding(dw, dtype))
    out["dbias"] = (db, R * U * g.abs().sum(0) + rounding(db, dtype))
    return out


# ---- routing
def scores64(logits, scores):
    z = logits.double()
    if scores == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    return torch.where(total == 0, torch.zeros_like(e), e / total)


def route64(logits, k, bias=None, scores="softmax", groups=1, top_groups=None, renormalize=False, scale=1.0):
    """(weights float64, experts), one row after the other."""
    logits, bias = logits.detach(), None if bias is None else bias.detach()
    rows, num = logits.shape
    top_groups = groups if top_groups is None else top_groups
    s = scores64(logits, scores)
    c = s if bias is None else s + bias.double()
    size = num // groups
    experts, weights = torch.full((rows, k), -1, dtype=torch.int64), torch.zeros(rows, k, dtype=torch.float64)
    order = lambda v: math.inf if v != v else v  # NaN first
    for r in range(rows):
        open_ = [e for e in range(num) if logits[r, e] != -math.inf and c[r, e] != -math.inf]
        if groups > 1:
            strength = {}
            for g in range(groups):
                best = sorted((float(c[r, e]) for e in open_ if e // size == g), key=order, reverse=True)[:2]
                if best:
                    strength[g] = order(sum(best))
            taken = sorted(strength, key=lambda g: (-strength[g], g))[:top_groups]
            open_ = [e for e in open_ if e // size in taken]
        ids = sorted(open_, key=lambda e: (-order(float(c[r, e])), e))[:k]
        total = sum(float(s[r, e]) for e in ids)
        for j, e in enumerate(ids):
            experts[r, j] = e
            v = float(s[r, e])
            weights[r, j] = scale * (v if not renormalize else 0.0 if total == 0 else v / total)
    return weights, experts


def weights_tol(w):
    return 2 * U * w.abs() + 2.0 ** -149  # 64-bit arithmetic, rounded once


def route_backward64(logits, experts, grad, scores="softmax", renormalize=False, scale=1.0):
    """dlogits and its tolerance.  Scores are exp of a difference rounded by U |z - top|, with a few units of its own and of the sum's
    (at most 16 + 6 links)."""
    s = scores64(logits, scores)
    there = experts >= 0
    at = experts.clamp(min=0)
    z = logits.double()
    if scores == "softmax":
        top = z.max(1, keepdim=True).values
        far = torch.where(s == 0, torch.zeros_like(s), (z - top).abs())
        r = (U * (far.max(1, keepdim=True).values * 2 + 40)).expand_as(s)
    else:
        r = U * (z.abs().clamp(max=200) + 16)
    worst = r.max(1, keepdim=True).values
    pick = torch.gather(s, 1, at) * there
    g = scale * grad.double() * there
    eg = 2 * U * g.abs()
    if renormalize:
        total = pick.sum(1, keepdim=True)
        total = torch.where(total == 0, torch.ones_like(total), total)
        mean = (g * pick).sum(1, keepdim=True) / total
        size = (g * pick).abs().sum(1, keepdim=True) / total
        ds = (g - mean) / total * there
        eg = (((2 * worst + 20 * U) * size + 4 * U * (g.abs() + mean.abs())) / total + (worst + 12 * U) * (g.abs() + mean.abs()) / total) * there
        g = ds
    dot = (g * pick).sum(1, keepdim=True)
    edot = ((eg + g.abs() * (worst + 12 * U)) * pick).sum(1, keepdim=True)
    d = torch.zeros_like(s).scatter_add_(1, at, g * there)
    ed = torch.zeros_like(s).scatter_add_(1, at, eg * there)
    if scores == "softmax":
        dz = s * (d - dot)
        tol = s * (ed + edot + (r + 4 * U) * (d.abs() + dot.abs()))
    else:
        dz = d * s * (1 - s)
        tol = (ed + d.abs() * (2 * r + 8 * U)) * s * (1 - s)
    dz = torch.where(s == 0, torch.zeros_like(dz), dz)
    return dz, tol + rounding(dz, logits.dtype)


def order_ref(experts, num):
    """(offsets, slots, sources) by lists."""
    flat = experts.reshape(-1).tolist()
    slots, sources, offsets = [-1] * len(flat), [], [0]
    by = [[] for _ in range(num)]
    for i, e in enumerate(flat):
        if 0 <= e < num:
            by[e].append(i)
    for e in range(num):
        for i in by[e]:
            slots[i] = len(sources)
            sources.append(i)
        offsets.append(len(sources))
    sources += [-1] * (len(flat) - len(sources))
    return (torch.tensor(offsets, dtype=torch.int64), torch.tensor(slots, dtype=torch.int32).view(experts.shape), torch.tensor(sources, dtype=torch.int32))


# ---- the experts' rows
def rows_ref(x, slots):
    """out in x's type; NaN in places without a source."""
    out = torch.full((slots.numel(), x.shape[1]), math.nan, dtype=torch.float64).to(x.dtype)
    for r in range(slots.shape[0]):
        for s in slots[r].tolist():
            if s >= 0:
                out[s] = x[r]
    return out


def combine64(y, slots, weights=None, residual=None, grad=None):
    """out, and with `grad` dy (NaN in places without a source) and dweights, each with its tolerance."""
    rows, k, n, dtype = slots.shape[0], slots.shape[1], y.shape[1], y.dtype
    there, at = (slots >= 0)[:, :, None], slots.clamp(min=0).long()
    yy = torch.where(there, y.double()[at], torch.zeros((), dtype=torch.float64))
    w = torch.ones(rows, k, dtype=torch.float64) if weights is None else weights.double()
    res = torch.zeros(rows, n, dtype=torch.float64) if residual is None else residual.double()
    terms = yy * w[:, :, None]
    out = terms.sum(1) + res
    result = dict(out=(out, (k + 2) * U * (terms.abs().sum(1) + res.abs()) + rounding(out, dtype)))
    if grad is None:
        return result
    g = grad.double()
    dy = torch.full((rows * k, n), math.nan, dtype=torch.float64)
    for r in range(rows):
        for j in range(k):
            if slots[r, j] >= 0:
                dy[slots[r, j].item()] = w[r, j] * g[r]
    dw = (yy * g[:, None, :]).sum(2)
    links = 80 + n // 16  # n / 16 terms a lane at the most, then six joins
    result["dy"] = (dy, U * dy.abs() + rounding(dy, dtype))
    result["dweights"] = (dw, links * U * (yy * g[:, None, :]).abs().sum(2) + 2.0 ** -149)
    return result


# ---- the loss
def loss64(x, w, labels, bias=None, ignore_index=-100, reduction="mean", grad=None):
    """loss, lse and, with `grad` (of the loss's shape), dx, dw and dbias, each with its tolerance.

    A logit is a sum of dim products in fp32 (twice dim + 2 units of sum |terms|, as for the products themselves).  lse: the largest error
    of a logit, the rounding of z - top in exp, and a sum with chains of at most 64 + classes / 256 links.  G: the errors of its exponent,
    its rounding to the type (fp16: scaled so that the largest share of the gradient is 2^13 or more, subnormal steps of 2^-25)."""
    dtype, (rows, d), V = x.dtype, x.shape, w.shape[0]
    counts = labels != ignore_index
    x = torch.where(counts[:, None], x.double(), torch.zeros((), dtype=torch.float64))
    w = w.double()
    b = torch.zeros(V, dtype=torch.float64) if bias is None else bias.double()
    z = x @ w.t() + b
    fin = torch.where(b == -math.inf, torch.zeros_like(b), b.abs())
    ez = 2 * (d + 2) * U * (x.abs() @ w.abs().t() + fin) + U * fin
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    top = z.max(1, keepdim=True).values
    far = torch.where(p == 0, torch.zeros_like(z), (z - top).abs())
    el = (p * (ez + 2 * U * far)).sum(1) + (80 + V / 256) * U + 6 * U * (lse.abs() + top[:, 0].abs())
    label = torch.where(counts, labels, torch.zeros_like(labels))[:, None]
    zl = z.gather(1, label)[:, 0]
    loss = torch.where(counts, lse - zl, torch.zeros_like(lse))
    eloss = torch.where(counts, el + ez.gather(1, label)[:, 0] + 4 * U * (zl.abs() + loss.abs()), torch.zeros_like(lse))
    n = int(counts.sum())
    share = 1.0 / max(n, 1) if reduction == "mean" else 1.0
    result = dict(lse=(torch.where(counts, lse, torch.zeros_like(lse)), torch.where(counts, el, torch.zeros_like(el))))
    if reduction == "none":
        result["loss"] = (loss, eloss)
    else:
        total = loss.sum() * share
        result["loss"] = (total, eloss.sum() * share + 4 * U * total.abs())
    if grad is None:
        return result
    g = torch.where(counts, grad.double() * share * torch.ones(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64))[:, None]
    hot = torch.zeros_like(p).scatter_(1, label, 1.0)
    G = (p - hot) * g
    ep = ez + el[:, None] + U * (2 * (z - lse[:, None]).abs().clamp(max=200) + 8)
    eG = g.abs() * (p * ep + 2 * U * (p + hot))
    if dtype != torch.float32:
        eG = eG + torch.finfo(dtype).eps / 2 * (G.abs() + eG) + (g.abs().max() * 2.0 ** -38 if dtype == torch.float16 else 2.0 ** -133)
    size = G.abs() + eG
    dx, dw, db = G @ w, G.t() @ x, G.sum(0)
    result["dx"] = (dx, eG @ w.abs() + 2 * (V + 2) * U * (size @ w.abs()) + rounding(dx, dtype))
    result["dw"] = (dw, eG.t() @ x.abs() + 2 * (rows + 2) * U * (size.t() @ x.abs()) + rounding(dw, dtype))
    result["dbias"] = (db, eG.sum(0) + 2 * (rows + 2) * U * size.sum(0) + rounding(db, dtype))
    return result


# ---- the router's gradient at any size of the scores
def route_backward_wide64(logits, experts, grad, scores="softmax", renormalize=False, scale=1.0):
    """dlogits and its tolerance from normalised weights by differences of logarithms, which no size of a score takes out of the range.  64-bit
    arithmetic, 2^-44 of the terms' sizes (some hundred roundings of 2^-53 each), rounded to fp32 and from there to the type."""
    z, there = logits.double(), experts >= 0
    at = experts.clamp(min=0)
    pick = lambda v: torch.where(there, torch.gather(v, 1, at), torch.full((), -math.inf, dtype=torch.float64))
    softplus = lambda v: v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    logs = z - torch.logsumexp(z, 1, keepdim=True) if scores == "softmax" else -softplus(-z)
    chosen = pick(logs)
    g = torch.where(there, scale * grad.double(), torch.zeros((), dtype=torch.float64))
    if renormalize:
        w = torch.softmax(chosen, 1).nan_to_num(0.0)
        t = w * (g - (g * w).sum(1, keepdim=True))
        size = w * (g.abs() + (g * w).abs().sum(1, keepdim=True))
    else:
        w = torch.exp(chosen)
        t, size = g * w, (g * w).abs()
    if scores == "sigmoid":
        rest = torch.where(there, torch.exp(-softplus(torch.gather(z, 1, at))), torch.zeros((), dtype=torch.float64))
        t, size = t * rest, size * rest
    dz, tol = (torch.zeros_like(z).scatter_add_(1, at, v) for v in (t, size))
    if scores == "softmax" and not renormalize:
        s, dot = torch.exp(logs), t.sum(1, keepdim=True)
        dz, tol = dz - s * dot, tol + s * size.sum(1, keepdim=True)
    return dz, 2.0 ** -44 * tol + rounding(dz, torch.float32) + (rounding(dz, logits.dtype) if logits.dtype != torch.float32 else 0)
