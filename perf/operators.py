"""Performance cases of the dense side of the library: the product behind the pooled rows (`tt_dense`, with one
weight or with a weight per group of rows) and the orthogonalised update (`tt_orthogonalize`, `tt_core_ortho_update`).

`listed()` are the named cases, `draw(rng)` gives another one of the same ranges, `prepare(case, seed)` makes what a
program holds before the call, `run(state)` is one pass, `work(case)` what the pass cannot do without, `exact(case,
seed)` the outputs from the definition in 64 bits.  Where `own` is false `run` computes the operators from elementary
torch operations in 32 bits, rounded once at the end; where it is true it makes the calls that a user makes.

  dense   z = x W^T + bias, y = act(z) + residual; in training also the gradients of x, W, bias and residual
  grouped the same with a weight and a bias for every group of rows; `offsets` holds the groups' first rows and the end
  ortho   X = G / (|G| + eps), five times X <- a X + (b A + c A^2) X with A = X X^T (mirrored for tall G): the
          Newton-Schulz iteration of the Muon optimiser (K. Jordan and others, 2024) with its published coefficients
  cores   m <- mu m + g, u = g + mu m; every slice of every core: G <- G - lr sqrt(max(1, rows / cols)) ortho(u)
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
LR, MOMENTUM = 1e-3, 0.95
MOST_FLOPS, MOST_BYTES = 5.6e11, 1.5e9  # a drawn case costs no more than the largest listed one


def listed():
    return [
        # Online serving of one sample: one pooled row (D = 128) projected to the width of the model above it.
        dict(name="dense_one_row", kind="dense", train=False, rows=1, k=128, n=512, dtype="f32", act="relu", residual=False, pad=0),
        # A single token through a square layer of a larger model: the weight is read once, nothing else counts.
        dict(name="dense_one_token", kind="dense", train=False, rows=1, k=4096, n=4096, dtype="bf16", act="none", residual=True, pad=0),
        # A small serving batch through a wide layer.
        dict(name="dense_serve_batch", kind="dense", train=False, rows=48, k=1024, n=4096, dtype="bf16", act="silu", residual=False, pad=0),
        # Batch inference, the largest product: compute bound on the matrix cores.
        dict(name="dense_infer_large", kind="dense", train=False, rows=16384, k=4096, n=4096, dtype="bf16", act="gelu", residual=True, pad=0),
        # Training of the projection behind one table at the batch of the multi-hot workload, in the bags' own precision.
        dict(name="dense_train_f32", kind="dense", train=True, rows=16384, k=128, n=512, dtype="f32", act="relu", residual=False, pad=0),
        # Odd sizes, a ragged batch, rows that are views into wider ones, half precision with a scaled loss.
        dict(name="dense_train_odd", kind="dense", train=True, rows=3001, k=479, n=513, dtype="f16", act="gelu", residual=True, pad=5),
        # 26 features' pooled rows, a matrix for every feature: serving, a few rows each, some features absent.
        dict(name="grouped_serve", kind="grouped", train=False, rows=100, groups=26, k=128, n=512, dtype="bf16", act="relu", residual=False, skew=1.0),
        # ... and training at the usual batch of 4096 bags a table, single precision as the bags give it.
        dict(name="grouped_train_f32", kind="grouped", train=True, rows=26 * 4096, groups=26, k=128, n=128, dtype="f32", act="none", residual=False, skew=0.0),
        # Experts: 64 weights, rows dealt very unevenly by a router, some experts without any.
        dict(name="grouped_train_experts", kind="grouped", train=True, rows=32768, groups=64, k=1024, n=1024, dtype="bf16", act="silu", residual=False, skew=1.2),
        # The update of all cores of the largest table (40 M rows, ranks 64): 1026 slices.
        dict(name="cores_40m", kind="cores", n1=342, n2=342, n3=342, d1=4, d2=8, d3=4, R1=64, R2=64),
        # The update of one projection in single precision.
        dict(name="ortho_projection", kind="ortho", batch=1, rows=512, cols=128, dtype="f32"),
        # The update of a large bfloat16 layer.
        dict(name="ortho_large", kind="ortho", batch=1, rows=4096, cols=2048, dtype="bf16"),
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
        kind = rng.choice(("dense", "dense", "grouped", "grouped", "ortho", "cores"))
        if kind == "dense":
            case = dict(kind=kind, train=rng.random() < 0.5, rows=_size(rng, 1, 65536), k=_size(rng, 16, 4096), n=_size(rng, 16, 4096),
                        dtype=rng.choice(tuple(DTYPES)), act=rng.choice(("none", "relu", "gelu", "silu", "sigmoid")),
                        residual=rng.random() < 0.5, pad=rng.choice((0, 0, 0, 5, 64)))
        elif kind == "grouped":
            case = dict(kind=kind, train=rng.random() < 0.6, rows=_size(rng, 16, 106496), groups=_log_int(rng, 2, 128), k=_size(rng, 32, 2048),
                        n=_size(rng, 32, 2048), dtype=rng.choice(tuple(DTYPES)), act=rng.choice(("none", "relu", "gelu", "silu", "sigmoid")),
                        residual=rng.random() < 0.3, skew=rng.choice((0.0, 0.6, 1.2)))
        elif kind == "ortho":
            case = dict(kind=kind, batch=_log_int(rng, 1, 64), rows=_size(rng, 16, 4096), cols=_size(rng, 16, 4096), dtype=rng.choice(tuple(DTYPES)))
        else:
            n = [_log_int(rng, 10, 342) for _ in range(3)]
            d = rng.choice(((4, 8, 4), (2, 2, 4), (4, 4, 4), (2, 4, 6)))
            R = rng.choice(((4, 4), (16, 16), (12, 20), (32, 32), (64, 64)))
            case = dict(kind=kind, n1=n[0], n2=n[1], n3=n[2], d1=d[0], d2=d[1], d3=d[2], R1=R[0], R2=R[1])
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _sizes(case):
    """Rows of every group: shares fall with a power of the group's rank, ranks in an order of their own; the last ones get nothing."""
    groups, rows = case["groups"], case["rows"]
    share = [(1.0 + g) ** -case["skew"] for g in range(groups)]
    if case["skew"]:
        share[-max(1, groups // 16):] = [0.0] * max(1, groups // 16)
    ends = [int(round(rows * sum(share[:g + 1]) / sum(share))) for g in range(groups)]
    sizes = [e - s for s, e in zip([0] + ends, ends)]
    step = next(s for s in range(groups // 2 + 1, 2 * groups + 2) if math.gcd(s, groups) == 1)
    return [sizes[g * step % groups] for g in range(groups)]


def _matrices(case):
    """(number, rows, columns) of the slices of the three cores."""
    return ((case["n1"], case["d1"], case["R1"]), (case["n2"], case["R1"], case["d2"] * case["R2"]), (case["n3"], case["R2"], case["d3"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    state = dict(case)
    if case["kind"] == "ortho":
        state["g"] = normal(case["batch"], case["rows"], case["cols"], std=1e-3).to(DTYPES[case["dtype"]])
        return state
    if case["kind"] == "cores":
        r = (1, case["R1"], case["R2"], 1)
        n, d = (case["n1"], case["n2"], case["n3"]), (case["d1"], case["d2"], case["d3"])
        numel = [r[k] * n[k] * d[k] * r[k + 1] for k in range(3)]
        state.update(n=n, d=d, r=r, cores=[normal(x, std=0.05) for x in numel], grads=[normal(x, std=1e-4) for x in numel],
                     momenta=[normal(x, std=1e-3) for x in numel])
        return state
    t, rows, k, n = DTYPES[case["dtype"]], case["rows"], case["k"], case["n"]
    pad = case.get("pad", 0)
    lead = (case["groups"],) if case["kind"] == "grouped" else ()
    # pooled rows, weights as they are initialised, gradients of a mean loss (half precision: of a scaled one)
    state["x"] = normal(rows, k + pad).to(t)[:, :k]
    state["w"] = normal(*lead, n, k, std=k ** -0.5).to(t)
    state["bias"] = normal(*lead, n, std=0.1).to(t)
    state["residual"] = normal(rows, n + pad).to(t)[:, :n] if case["residual"] else None
    if case["kind"] == "grouped":
        state["sizes"] = _sizes(case)
        state["offsets"] = torch.tensor([0] + state["sizes"], dtype=torch.int64).cumsum(0).cuda()
    if case["train"]:
        state["gy"] = normal(rows, n, std=rows ** -0.5 if case["dtype"] == "f16" else 1.0 / rows).to(t)
        for name in ("x", "w", "bias", "residual"):
            if state[name] is not None:
                state[name].requires_grad_(True)
    else:
        state["out"] = torch.empty(rows, n, dtype=t, device="cuda")
    return state


def _act(z, act):
    if act == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return 1 / (1 + torch.exp(-z)) if act == "sigmoid" else z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s)) if act == "silu" else s * (1 - s)


def _ortho(g):
    """Newton-Schulz steps on [batch, rows, cols] in 32 bits (the norm in 64)."""
    x = g.float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x * (1 / (x.double().square().sum((1, 2), keepdim=True).sqrt() + EPS)).float()
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        A = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * A + c * torch.bmm(A, A), x)
    return x.transpose(1, 2) if tall else x


def _slices(core, k, s):
    """Core k as [slices, rows, columns] (a view where the core's order allows it)."""
    c = core.view(s["r"][k], s["n"][k], s["d"][k], s["r"][k + 1])
    return c[0] if k == 0 else c.transpose(0, 1).reshape(s["n"][k], s["r"][k], s["d"][k] * s["r"][k + 1])


def _unslice(x, k, s):
    return x.reshape(-1) if k == 0 else x.transpose(0, 1).reshape(-1)


def _run_cores(s):
    for k in range(3):
        core, g, m = s["cores"][k], s["grads"][k], s["momenta"][k]
        m.mul_(MOMENTUM).add_(g)
        u = _slices(g + MOMENTUM * m, k, s)
        core.sub_(LR * math.sqrt(max(1.0, u.shape[1] / u.shape[2])) * _unslice(_ortho(u), k, s))
    return s["cores"] + s["momenta"]


def _run_product(s):
    t = s["x"].dtype
    x, w, bias = s["x"].detach().float(), s["w"].detach().float(), s["bias"].detach().float()
    res = s["residual"].detach().float() if s["residual"] is not None else None
    gy = s["gy"].float() if s["train"] else None
    if s["kind"] == "dense":
        z = x @ w.t() + bias
    else:
        xs = x.split(s["sizes"])
        z = torch.cat([xg @ wg.t() + bg for xg, wg, bg in zip(xs, w, bias)])
    y = _act(z, s["act"])
    y = (y if res is None else y + res).to(t)
    if not s["train"]:
        return y
    gz = gy if s["act"] == "none" else gy * _act_grad(z, s["act"])
    if s["kind"] == "dense":
        gx, gw, gb = gz @ w, gz.t() @ x, gz.sum(0)
    else:
        gs = gz.split(s["sizes"])
        gx = torch.cat([g @ wg for g, wg in zip(gs, w)])
        gw = torch.stack([g.t() @ xg for g, xg in zip(gs, xs)])
        gb = torch.stack([g.sum(0) for g in gs])
    out = [y, gx.to(t), gw.to(t), gb.to(t)]
    return out if res is None else out + [gy.to(t)]


def run(state):
    s = state
    if not own:
        if s["kind"] == "ortho":
            return _ortho(s["g"]).to(s["g"].dtype)
        return _run_cores(s) if s["kind"] == "cores" else _run_product(s)
    import paper_2507_14668_amd as tt
    if s["kind"] == "ortho":
        return tt.tt_orthogonalize(s["g"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
    if s["kind"] == "cores":
        table = tt.Table(s["n"][0] * s["n"][1] * s["n"][2], s["n"], s["d"], s["r"], s["cores"])
        tt.tt_core_ortho_update(table, s["grads"], s["momenta"], LR, momentum=MOMENTUM, nesterov=True, steps=STEPS,
                                coefficients=COEFFICIENTS, eps=EPS)
        return s["cores"] + s["momenta"]
    offsets = s.get("offsets")
    if not s["train"]:
        return tt.tt_dense_forward(s["x"], s["w"], s["bias"], s["residual"], s["act"], offsets=offsets, out=s["out"])
    y = tt.tt_dense(s["x"], s["w"], s["bias"], s["residual"], s["act"], offsets=offsets)
    leaves = [s["x"], s["w"], s["bias"]] + ([s["residual"]] if s["residual"] is not None else [])
    return [y.detach()] + list(torch.autograd.grad(y, leaves, s["gy"]))


def _ortho_flops(batch, rows, cols):
    """The cheaper of two ways, symmetric products by half: on the matrix itself, or on the products of its short side."""
    m, n = min(rows, cols), max(rows, cols)
    return batch * min(STEPS * (m * m * n + m ** 3 + 2 * m * m * n), 3 * m * m * n + STEPS * 4 * m ** 3)


def work(case):
    if case["kind"] == "ortho":
        es = 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * es * case["batch"] * case["rows"] * case["cols"], "flops": _ortho_flops(case["batch"], case["rows"], case["cols"])}
    if case["kind"] == "cores":
        mats = _matrices(case)  # read cores, gradients and momenta, write cores and momenta
        return {"bytes": sum(5 * 4 * b * r * c for b, r, c in mats), "flops": sum(_ortho_flops(*m) for m in mats)}
    rows, k, n = case["rows"], case["k"], case["n"]
    es = 4 if case["dtype"] == "f32" else 2
    weights = case.get("groups", 1) * (n * k + n)
    fwd = rows * k + weights + rows * n * (2 if case["residual"] else 1)
    if not case["train"]:
        return {"bytes": es * fwd, "flops": 2 * rows * k * n}
    # the forward; the output's gradient read; the gradients of x, weights and biases written
    return {"bytes": es * (fwd + rows * n + rows * k + weights), "flops": 6 * rows * k * n}


def _exact_ortho(g):
    """[batch, rows, cols] in 64 bits, with the products on whichever side is the shorter."""
    g = g.double()
    x = g / (torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True) + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        xt = x.mT.contiguous()
        if x.shape[1] <= x.shape[2]:
            A = x @ xt
            x = a * x + b * (A @ x) + c * (A @ (A @ x))
        else:
            A = xt @ x
            x = a * x + b * (x @ A) + c * ((x @ A) @ A)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ortho":
        return _exact_ortho(s["g"])
    if case["kind"] == "cores":
        cores, momenta = [], []
        for k, (num, rows, cols) in enumerate(_matrices(case)):
            G, g, m = (s[name][k].double().view(s["r"][k], num, -1) for name in ("cores", "grads", "momenta"))
            m = MOMENTUM * m + g
            u = (g + MOMENTUM * m).permute(1, 0, 2).reshape(num, rows, cols)
            O = _exact_ortho(u).reshape(num, s["r"][k], -1).permute(1, 0, 2)
            cores.append((G - LR * max(1.0, rows / cols) ** 0.5 * O).reshape(-1))
            momenta.append(m.reshape(-1))
        return cores + momenta
    x, w, bias = (s[name].detach().double() for name in ("x", "w", "bias"))
    sizes = s.get("sizes", [case["rows"]])
    ws, bs = (w, bias) if case["kind"] == "grouped" else (w[None], bias[None])
    parts, at = [], 0
    for g, size in enumerate(sizes):
        xg = x[at:at + size]
        z = torch.addmm(bs[g], xg, ws[g].t())
        if case["act"] == "relu":
            y, slope = z.clamp(min=0), (z > 0).double()
        elif case["act"] == "gelu":
            cdf = 0.5 * torch.erfc(-z / 2 ** 0.5)
            y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
        elif case["act"] == "silu":
            sg = torch.sigmoid(z)
            y, slope = z * sg, sg + z * sg * (1 - sg)
        elif case["act"] == "sigmoid":
            y = torch.sigmoid(z)
            slope = y * (1 - y)
        else:
            y, slope = z, torch.ones_like(z)
        if s["residual"] is not None:
            y = y + s["residual"].detach()[at:at + size].double()
        if case["train"]:
            gz = s["gy"][at:at + size].double() * slope
            parts.append((y, gz @ ws[g], gz.t() @ xg, gz.sum(0)))
        else:
            parts.append((y,))
        at += size
    y = torch.cat([p[0] for p in parts])
    if not case["train"]:
        return y
    gw, gb = torch.stack([p[2] for p in parts]), torch.stack([p[3] for p in parts])
    if case["kind"] == "dense":
        gw, gb = gw[0], gb[0]
    out = [y, torch.cat([p[1] for p in parts]), gw, gb]
    return out if s["residual"] is None else out + [s["gy"].double()]
