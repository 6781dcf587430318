"""Performance cases of what a model puts on top of the pooled rows: layer norm, a router with the experts' rows it
deals, and softmax cross entropy over a large catalogue.

`listed()` are the named cases, `draw(rng)` gives another one of the same ranges, `prepare(case, seed)` makes what a
program holds before the call, `run(state)` is one pass, `work(case)` what the pass cannot do without, `exact(case,
seed)` the outputs from the definition in 64 bits.  Where `own` is false `run` computes the operators from elementary
torch operations, rounded once at the end; where it is true it makes the calls that a user makes.

  norm   y = (x - mean) / sqrt(var + eps) * weight + bias, row by row; in training the gradients of x, weight and bias
  route  s = softmax or sigmoid of the logits, c = s + bias; of `groups` equal groups of experts the `top_groups` with the
         largest sum of their two best c; of their experts the k with the largest c, largest first, ties to the lowest number;
         weights scale * s, divided by their sum if `renorm`.  An expert whose logit is -infinity is not chosen; where fewer
         than k are left the numbers are -1 and the weights 0.  Then the rows in the experts' order: `offsets` where each
         expert's start, `slots` the place of each (row, choice), `sources` the (row, choice) of each place
  rows   the rows of x in the experts' order; out = residual + sum over a row's choices of weight * y[slot]
  loss   logsumexp(x W^T + bias) - (x W^T + bias)[label], the mean over rows with a label in training, row by row without
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
IGNORED = -100
MOST_FLOPS, MOST_BYTES = 6.6e12, 1.2e9  # a drawn case costs no more than the largest listed one


def listed():
    return [
        # Online serving: one sample's projected row (128 -> 512) before the layers above it.
        dict(name="norm_one_row", kind="norm", train=False, rows=1, n=512, dtype="bf16", pad=0),
        # Training on the pooled rows of 26 tables of 4096 bags, in the bags' own width and precision.
        dict(name="norm_train_pooled", kind="norm", train=True, rows=26 * 4096, n=128, dtype="f32", pad=0),
        # Training of a wide layer, rows that are views into wider ones.
        dict(name="norm_train_wide", kind="norm", train=True, rows=16384, n=4096, dtype="bf16", pad=64),
        # One sample is sent to two of 64 experts.
        dict(name="route_one_row", kind="route", train=False, rows=1, experts=64, k=2, scores="softmax", bias=False, groups=1, top_groups=1,
             renorm=True, scale=1.0, dtype="f32", masked=False),
        # An odd batch with padding in it, an expert for each of 26 features, some of them masked, half-precision logits.
        dict(name="route_odd", kind="route", train=True, rows=3001, experts=26, k=3, scores="softmax", bias=True, groups=1, top_groups=1,
             renorm=False, scale=1.0, dtype="bf16", masked=True),
        # A large training batch over many small experts: sigmoid scores, a bias that balances them, eight groups of which four are taken.
        dict(name="route_train_groups", kind="route", train=True, rows=16384, experts=256, k=8, scores="sigmoid", bias=True, groups=8,
             top_groups=4, renorm=True, scale=2.5, dtype="f32", masked=False),
        # A serving batch's rows to their experts and back.
        dict(name="rows_serve", kind="rows", train=False, rows=48, experts=64, k=2, n=1024, dtype="bf16", residual=True, masked=False, skew=0.5),
        # Training: the rows of a large batch to four experts each, with padding, and their gradients.
        dict(name="rows_train", kind="rows", train=True, rows=16384, experts=64, k=4, n=1024, dtype="bf16", residual=True, masked=True, skew=1.0),
        # A small catalogue in the bags' own width and precision, training.
        dict(name="loss_small", kind="loss", train=True, rows=512, d=128, v=10000, dtype="f32", bias=True, ignored=0.0),
        # Scoring a ragged batch against a catalogue: losses only, half precision, an odd width.
        dict(name="loss_odd", kind="loss", train=False, rows=1001, d=479, v=50001, dtype="f16", bias=False, ignored=0.1),
        # The next item out of half a million, training with a correction for how often items are seen.
        dict(name="loss_items", kind="loss", train=True, rows=4096, d=128, v=500001, dtype="bf16", bias=True, ignored=0.1),
        # A wide layer on a large vocabulary: compute bound on the matrix cores.
        dict(name="loss_wide", kind="loss", train=True, rows=4096, d=4096, v=65536, dtype="bf16", bias=False, ignored=0.02),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Log-uniform, a third each: any number, a multiple of 8, a multiple of 64."""
    v = _log_int(rng, lo, hi)
    m = rng.choice((1, 8, 64))
    return max(lo, v // m * m)


def draw(rng):
    """One more case: kinds in equal shares, sizes log-uniform over the ranges of the listed cases."""
    while True:
        kind = rng.choice(("norm", "route", "rows", "loss"))
        dtype = rng.choice(tuple(DTYPES))
        if kind == "norm":
            case = dict(kind=kind, train=rng.random() < 0.6, rows=_size(rng, 1, 131072), n=_size(rng, 16, 8192), dtype=dtype,
                        pad=rng.choice((0, 0, 5, 64)))
        elif kind == "route":
            size, groups = _log_int(rng, 2, 64), rng.choice((1, 1, 2, 4, 8))
            top = rng.randint(1, groups)
            case = dict(kind=kind, train=rng.random() < 0.6, rows=_size(rng, 1, 65536), experts=groups * size, k=rng.randint(1, min(8, top * size)),
                        scores=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5, groups=groups, top_groups=top,
                        renorm=rng.random() < 0.7, scale=rng.choice((1.0, 2.5)), dtype=dtype, masked=rng.random() < 0.3)
        elif kind == "rows":
            experts = _log_int(rng, 2, 256)
            case = dict(kind=kind, train=rng.random() < 0.6, rows=_size(rng, 1, 32768), experts=experts, k=rng.randint(1, min(8, experts)),
                        n=_size(rng, 16, 4096), dtype=dtype, residual=rng.random() < 0.5, masked=rng.random() < 0.5,
                        skew=rng.choice((0.0, 0.5, 1.0)))
        else:
            case = dict(kind=kind, train=rng.random() < 0.6, rows=_size(rng, 1, 16384), d=_size(rng, 16, 4096), v=_size(rng, 64, 500001),
                        dtype=dtype, bias=rng.random() < 0.5, ignored=rng.choice((0.0, 0.02, 0.1)))
            if case["rows"] * case["v"] > 4096 * 500001:
                continue
        w = work(case)
        # single precision has a tenth of the matrix cores' rate
        if w["flops"] * (8 if case["dtype"] == "f32" else 1) <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _order(experts, num):
    """(offsets, slots, sources) of the choices [rows, k], those of one expert in the order of the rows; -1 goes nowhere."""
    flat = experts.reshape(-1)
    key = torch.where(flat < 0, torch.full_like(flat, num), flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(num + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([counts.new_zeros(1), counts[:num].cumsum(0)])
    slots = torch.empty_like(order)
    slots[order] = torch.arange(order.numel(), device=flat.device)
    slots = torch.where(flat < 0, torch.full_like(slots, -1), slots).view_as(experts)
    sources = torch.where(torch.arange(order.numel(), device=flat.device) < offsets[num], order, torch.full_like(order, -1))
    return offsets, slots.int(), sources.int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    state, t, rows = dict(case), DTYPES[case["dtype"]], case["rows"]
    if case["kind"] == "norm":
        n = case["n"]
        # activations with an offset of their own a row, weights after some training
        state["x"] = (normal(rows, n + case["pad"], std=2.0) + normal(rows, 1)).to(t)[:, :n]
        state["weight"] = (1 + normal(n, std=0.2)).to(t)
        state["bias"] = normal(n, std=0.1).to(t)
        if case["train"]:
            state["gy"] = normal(rows, n).to(t)
            for name in ("x", "weight", "bias"):
                state[name].requires_grad_(True)
        return state
    if case["kind"] == "loss":
        d, v = case["d"], case["v"]
        # rows after a norm, a matrix that gives logits of a deviation of 2, labels that favour the first entries, as sorted by how often they are seen
        state["x"] = normal(rows, d).to(t)
        state["w"] = normal(v, d, std=2.0 * d ** -0.5).to(t)
        state["b"] = (-0.2 * torch.log1p(torch.arange(v, device="cuda").float())).to(t) if case["bias"] else None
        state["labels"] = (v * torch.rand(rows, generator=gen, device="cuda").double() ** 3).long().clamp(max=v - 1)
        state["labels"][torch.rand(rows, generator=gen, device="cuda") < case["ignored"]] = IGNORED
        if case["train"]:
            # half precision is trained with a scaled loss
            state["gy"] = torch.tensor(float(rows) if case["dtype"] == "f16" else 1.0, device="cuda")
            for name in ("x", "w", "b"):
                if state[name] is not None:
                    state[name].requires_grad_(True)
        return state
    experts, k = case["experts"], case["k"]
    if case["kind"] == "route":
        # logits as a projection gives them, experts that are liked more than others
        logits = normal(rows, experts, std=1.5) + normal(experts, std=0.5)
        if case["masked"]:
            logits[torch.rand(rows, experts, generator=gen, device="cuda") < 0.1] = -math.inf
            logits[torch.rand(rows, generator=gen, device="cuda") < 0.05] = -math.inf  # padding
        state["logits"] = logits.to(t)
        # a balancing bias moves in steps
        state["b"] = torch.randint(-50, 51, (experts,), generator=gen, device="cuda").float() * 1e-3 if case["bias"] else None
        if case["train"]:
            state["gw"] = normal(rows, k)
            state["logits"].requires_grad_(True)
        return state
    n = case["n"]
    likes = -case["skew"] * torch.log1p(torch.arange(experts, device="cuda").float())
    noise = -torch.log(-torch.log(torch.rand(rows, experts, generator=gen, device="cuda").clamp(1e-7, 1 - 1e-6)))
    chosen = torch.sort(noise + likes, dim=1, descending=True, stable=True).indices[:, :k].contiguous()
    weights = torch.softmax(normal(rows, k), 1)
    if case["masked"]:
        none = torch.rand(rows, generator=gen, device="cuda") < 0.05
        chosen[none], weights[none] = -1, 0.0
    state.update(chosen=chosen, weights=weights, x=normal(rows, n).to(t), y=normal(rows * k, n).to(t), residual=normal(rows, n).to(t) if case["residual"] else None)
    state["offsets"], state["slots"], state["sources"] = _order(chosen, experts)
    if case["train"]:
        state["gxs"], state["gout"] = normal(rows * k, n).to(t), normal(rows, n).to(t)
        for name in ("x", "y", "weights", "residual"):
            if state[name] is not None:
                state[name].requires_grad_(True)
    return state


def _run_norm(s):
    t = s["x"].dtype
    x, w, b = s["x"].detach().float(), s["weight"].detach().float(), s["bias"].detach().float()
    xc = x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh = xc * rstd
    y = (xh * w + b).to(t)
    if not s["train"]:
        return y
    g = s["gy"].float()
    h = g * w
    dx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    return [y, dx.to(t), (g * xh).sum(0).to(t), g.sum(0).to(t)]


def _run_route(s):
    # in 64 bits: which experts are taken hangs on scores that lie next to each other
    z = s["logits"].detach().double()
    rows, num = z.shape
    masked = z == -math.inf
    if s["scores"] == "softmax":
        top = z.max(1, keepdim=True).values
        e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = e.sum(1, keepdim=True)
        score = e / torch.where(total == 0, torch.ones_like(total), total)
    else:
        score = 1 / (1 + torch.exp(-z))
    c = score if s["b"] is None else score + s["b"].double()
    c = torch.where(masked, torch.full_like(c, -math.inf), c)
    if s["groups"] > 1:
        by = c.view(rows, s["groups"], -1)
        best = torch.sort(by, dim=2, descending=True).values[:, :, :2]
        best = torch.where(best == -math.inf, torch.zeros_like(best), best).sum(2)
        best = torch.where((by == -math.inf).all(2), torch.full_like(best, -math.inf), best)
        taken = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        keep = torch.zeros(rows, s["groups"], dtype=torch.bool, device=z.device).scatter_(1, taken, True)
        c = torch.where(keep[:, :, None], by, torch.full_like(by, -math.inf)).reshape(rows, num)
    order = torch.sort(c, dim=1, descending=True, stable=True)
    chosen = order.indices[:, :s["k"]]
    there = order.values[:, :s["k"]] != -math.inf
    picked = torch.where(there, torch.gather(score, 1, chosen), torch.zeros((), dtype=z.dtype, device=z.device))
    total = picked.sum(1, keepdim=True)
    total = torch.where(total == 0, torch.ones_like(total), total)
    weights = s["scale"] * (picked / total if s["renorm"] else picked)
    experts = torch.where(there, chosen, torch.full_like(chosen, -1))
    out = [weights.float(), experts, *_order(experts, num)]
    if not s["train"]:
        return out
    g = s["scale"] * s["gw"].double() * there
    if s["renorm"]:
        g = (g - (g * picked).sum(1, keepdim=True) / total) / total * there
    ds = torch.zeros_like(score).scatter_add_(1, chosen, g)
    dz = score * (ds - (ds * score).sum(1, keepdim=True)) if s["scores"] == "softmax" else ds * score * (1 - score)
    return out + [dz.to(s["logits"].dtype)]


def _run_rows(s):
    t, rows, k = s["x"].dtype, s["rows"], s["k"]
    src, slots = s["sources"].long(), s["slots"].long()
    some, there = (src >= 0)[:, None], (slots >= 0)[:, :, None]
    row, slot = src.clamp(min=0) // k, slots.clamp(min=0)
    x, y, w = s["x"].detach(), s["y"].detach(), s["weights"].detach()
    xs = torch.where(some, x[row], torch.zeros((), dtype=t, device=x.device))
    picked = torch.where(there, y[slot].float(), torch.zeros((), device=x.device))
    out = (picked * w[:, :, None]).sum(1)
    out = (out if s["residual"] is None else out + s["residual"].detach().float()).to(t)
    if not s["train"]:
        return [xs, out]
    g = s["gout"].float()
    dx = torch.where(there, s["gxs"][slot].float(), torch.zeros((), device=x.device)).sum(1).to(t)
    dy = torch.where(some, g[row] * w.reshape(-1)[src.clamp(min=0)][:, None], torch.zeros((), device=x.device)).to(t)
    dw = (picked * g[:, None, :]).sum(2)
    grads = [dx, dy, dw]
    return [xs, out] + (grads if s["residual"] is None else grads + [s["gout"]])


def _run_loss(s):
    t = s["x"].dtype
    x, w, labels = s["x"].detach().float(), s["w"].detach().float(), s["labels"]
    z = x @ w.t()
    if s["b"] is not None:
        z += s["b"].detach().float()
    there = labels != IGNORED
    label = labels.clamp(min=0)[:, None]
    top = z.max(1, keepdim=True).values
    of_label = z.gather(1, label)
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    losses = torch.where(there, (top + torch.log(total) - of_label)[:, 0], torch.zeros((), device=x.device))
    if not s["train"]:
        return losses
    count = there.sum().clamp(min=1)
    loss = losses.sum() / count
    g = (there * (s["gy"] / count))[:, None]
    G = e.mul_(g / total)
    G.scatter_add_(1, label, -g)
    grads = [(G @ w).to(t), (G.t() @ x).to(t)] + ([] if s["b"] is None else [G.sum(0).to(t)])
    return [loss] + grads


def run(state):
    s = state
    if not own:
        return {"norm": _run_norm, "route": _run_route, "rows": _run_rows, "loss": _run_loss}[s["kind"]](s)
    import paper_2507_14668_amd as tt
    if s["kind"] == "norm":
        y = tt.tt_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
        if not s["train"]:
            return y
        return [y.detach()] + list(torch.autograd.grad(y, [s["x"], s["weight"], s["bias"]], s["gy"]))
    if s["kind"] == "route":
        r = tt.tt_route(s["logits"], s["k"], bias=s["b"], scores=s["scores"], groups=s["groups"], top_groups=s["top_groups"],
                        renormalize=s["renorm"], scale=s["scale"])
        out = [r.weights.detach(), r.experts, r.offsets, r.slots, r.sources]
        return out + list(torch.autograd.grad(r.weights, [s["logits"]], s["gw"])) if s["train"] else out
    if s["kind"] == "rows":
        r = tt.Routes(s["weights"], s["chosen"], s["offsets"], s["slots"], s["sources"])
        xs = tt.tt_expert_rows(s["x"], r)
        out = tt.tt_expert_combine(s["y"], r, residual=s["residual"])
        if not s["train"]:
            return [xs, out]
        leaves = [s["x"], s["y"], s["weights"]] + ([] if s["residual"] is None else [s["residual"]])
        return [xs.detach(), out.detach()] + list(torch.autograd.grad([xs, out], leaves, [s["gxs"], s["gout"]]))
    if not s["train"]:
        return tt.tt_cross_entropy(s["x"], s["w"], s["labels"], s["b"], ignore_index=IGNORED, reduction="none")
    loss = tt.tt_cross_entropy(s["x"], s["w"], s["labels"], s["b"], ignore_index=IGNORED, reduction="mean")
    leaves = [s["x"], s["w"]] + ([] if s["b"] is None else [s["b"]])
    return [loss.detach()] + list(torch.autograd.grad(loss, leaves, s["gy"]))


def work(case):
    rows, es = case["rows"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        n = case["n"]
        if not case["train"]:
            return {"bytes": es * (2 * rows * n + 2 * n), "flops": 8 * rows * n}
        # x and weight once, y written; the output's gradient read, the gradients of x, weight and bias written
        return {"bytes": es * (4 * rows * n + 4 * n), "flops": 20 * rows * n}
    if case["kind"] == "route":
        num, k = case["experts"], case["k"]
        # logits (and bias) read; weights, numbers, slots and sources of the choices and the offsets written
        bytes_ = es * rows * num + 4 * num * case["bias"] + rows * k * (4 + 8 + 4 + 4) + 8 * (num + 1)
        if case["train"]:
            bytes_ += 4 * rows * k + es * rows * num
        return {"bytes": bytes_, "flops": (20 + 8 * case["train"]) * rows * num}
    if case["kind"] == "rows":
        n, k = case["n"], case["k"]
        # there: x read, its rows written; back: y, weights (and the residual) read, out written
        elements = (1 + k) * rows * n + (k + 1 + case["residual"]) * rows * n
        index = rows * k * (4 + 4 + 4)
        if case["train"]:  # there: the rows' gradient read, x's written; back: out's gradient read, y's, the weights' (and the residual's) written
            elements += (k + 1) * rows * n + (1 + k + case["residual"]) * rows * n
            index += rows * k * 4
        return {"bytes": es * elements + index, "flops": (4 if case["train"] else 1) * 2 * rows * k * n}
    d, v = case["d"], case["v"]
    params = v * d + v * case["bias"]
    if not case["train"]:
        return {"bytes": es * (rows * d + params) + 12 * rows, "flops": 2 * rows * d * v}
    return {"bytes": 2 * es * (rows * d + params) + 8 * rows, "flops": 6 * rows * d * v}


def _exact_norm(s):
    x, w, b = (s[name].detach().double() for name in ("x", "weight", "bias"))
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    sd = (var + EPS).sqrt()
    y = torch.addcmul(b, (x - mean) / sd, w)
    if not s["train"]:
        return y
    g = s["gy"].double()
    xh = (x - mean) / sd
    h = g * w
    n = x.shape[1]
    dx = (n * h - h.sum(1, keepdim=True) - xh * (h * xh).sum(1, keepdim=True)) / (n * sd)
    return [y, dx, torch.einsum("rn,rn->n", g, xh), g.sum(0)]


def _exact_route(s):
    """By counting: an expert's place is the number of experts that come before it."""
    z, num, k, groups = s["logits"].detach().double(), s["experts"], s["k"], s["groups"]
    chosen, weights, grads = [], [], []

    def places(c):  # of each column, among the columns
        at = torch.arange(c.shape[1], device=c.device)
        first = (c[:, None, :] > c[:, :, None]) | ((c[:, None, :] == c[:, :, None]) & (at[None, None, :] < at[None, :, None]))
        return first.sum(2)

    for lo in range(0, z.shape[0], 1024):
        part = z[lo:lo + 1024]
        if s["scores"] == "softmax":
            score = torch.nan_to_num(torch.softmax(part, 1), nan=0.0)
        else:
            score = torch.sigmoid(part)
        c = score + (s["b"].double() if s["b"] is not None else 0)
        c[part == -math.inf] = -math.inf
        if groups > 1:
            by = c.unflatten(1, (groups, -1))
            two = by.topk(min(2, by.shape[2]), dim=2).values
            strength = two.clamp(min=-1e9).sum(2) if by.shape[2] == 1 else two[:, :, 0] + torch.where(two[:, :, 1] == -math.inf, 0.0, two[:, :, 1])
            strength[(by == -math.inf).all(2)] = -math.inf
            c = by.masked_fill((places(strength) >= s["top_groups"])[:, :, None], -math.inf).flatten(1)
        place = places(c)
        taken = (place < k) & (c != -math.inf)
        row, col = taken.nonzero(as_tuple=True)
        ids = torch.full((part.shape[0], k), -1, dtype=torch.int64, device=z.device)
        ids[row, place[row, col]] = col
        sel = score * taken
        norm = sel.sum(1, keepdim=True)
        factor = s["scale"] / torch.where(norm == 0, 1.0, norm) if s["renorm"] else torch.full_like(norm, s["scale"])
        w = torch.zeros(part.shape[0], k, dtype=torch.float64, device=z.device)
        w[row, place[row, col]] = (sel * factor)[row, col]
        chosen.append(ids)
        weights.append(w)
        if s["train"]:
            up = torch.zeros_like(score)
            up[row, col] = s["gw"][lo:lo + 1024].double()[row, place[row, col]]
            if s["renorm"]:
                up = up - (up * sel).sum(1, keepdim=True) / torch.where(norm == 0, 1.0, norm)
            up = up * taken * factor
            grads.append(score * up - score * (score * up).sum(1, keepdim=True) if s["scores"] == "softmax" else up * score * (1 - score))
    ids = torch.cat(chosen)
    flat = ids.reshape(-1)
    offsets, slots, sources = [0], torch.full_like(flat, -1), torch.full_like(flat, -1)
    for e in range(num):
        at = (flat == e).nonzero()[:, 0]
        slots[at] = torch.arange(offsets[-1], offsets[-1] + at.numel(), device=z.device)
        sources[offsets[-1]:offsets[-1] + at.numel()] = at
        offsets.append(offsets[-1] + at.numel())
    out = [torch.cat(weights), ids, torch.tensor(offsets, device=z.device), slots.view_as(ids).int(), sources.int()]
    return out + [torch.cat(grads)] if s["train"] else out


def _exact_rows(s):
    rows, k, n = s["rows"], s["k"], s["n"]
    x, y, w = (s[name].detach().double() for name in ("x", "y", "weights"))
    xs = torch.zeros(rows * k, n, dtype=torch.float64, device=x.device)
    out = torch.zeros_like(x) if s["residual"] is None else s["residual"].detach().double()
    if s["train"]:
        g, gxs = s["gout"].double(), s["gxs"].double()
        dx, dy, dw = torch.zeros_like(x), torch.zeros_like(xs), torch.zeros_like(w)
    for j in range(k):
        row = (s["slots"][:, j] >= 0).nonzero()[:, 0]
        slot = s["slots"][row, j].long()
        xs[slot] = x[row]
        out[row] += w[row, j, None] * y[slot]
        if s["train"]:
            dx[row] += gxs[slot]
            dy[slot] = w[row, j, None] * g[row]
            dw[row, j] = (g[row] * y[slot]).sum(1)
    if not s["train"]:
        return [xs, out]
    return [xs, out, dx, dy, dw] + ([] if s["residual"] is None else [g])


def _exact_loss(s):
    x, w, labels = s["x"].detach().double(), s["w"].detach().double(), s["labels"]
    b = None if s["b"] is None else s["b"].detach().double()
    there = labels != IGNORED
    losses, dw, db, dx = [], torch.zeros_like(w) if s["train"] else None, None if b is None else torch.zeros_like(b), []
    g = float(s["gy"]) / max(1, int(there.sum())) if s["train"] else 0.0
    step = max(1, (1 << 28) // w.shape[0])
    for lo in range(0, x.shape[0], step):
        xp, yes = x[lo:lo + step], there[lo:lo + step]
        z = xp @ w.t() if b is None else torch.addmm(b, xp, w.t())
        logp = torch.log_softmax(z, 1)
        at = yes.nonzero()[:, 0]
        loss = torch.zeros(xp.shape[0], dtype=torch.float64, device=x.device)
        loss[at] = -logp[at, labels[lo:lo + step][at]]
        losses.append(loss)
        if s["train"]:
            p = logp.exp_()
            p[at, labels[lo:lo + step][at]] -= 1
            p *= (yes * g)[:, None]
            dx.append(p @ w)
            dw += p.t() @ xp
            if b is not None:
                db += p.sum(0)
    losses = torch.cat(losses)
    if not s["train"]:
        return losses
    return [losses.sum() / max(1, int(there.sum())), torch.cat(dx), dw] + ([] if b is None else [db])


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "rows": _exact_rows, "loss": _exact_loss}[case["kind"]](s)
