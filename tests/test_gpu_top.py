"""Layer norm, routing, the experts' rows and the softmax loss on the GPU: values against 64 bits over sizes, types and layouts; autograd,
modules, a run of them together, streams, graphs, reproducibility and refusals."""
import math

import pytest
import torch

import top_ref as ref
from test_top_emulation import FAR_ROUTES, LARGE, LOSSES, ROUTES, far_rows, large_logits, large_logits64, routed, stats_loss, sure_rows, sure_rows64

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def tt():
    import paper_2507_14668_amd as tt
    return tt


def put(t, pad=0, shift=0):
    """t on the GPU, in rows `pad` longer and `shift` elements behind an aligned address."""
    if t is None:
        return None
    wide = (*t.shape[:-1], t.shape[-1] + pad)
    flat = torch.empty(math.prod(wide) + shift, dtype=t.dtype, device="cuda")[shift:].view(wide)
    view = flat[..., :t.shape[-1]]
    view.copy_(t)
    return view


def randn(gen, *s, std=1.0, dtype=F32):
    return (torch.randn(*s, generator=gen) * std).to(dtype)


def cpu(*ts):
    return [None if t is None else t.detach().cpu() for t in ts]


def check(got, pair, what):
    ref.check(got.detach().cpu(), *pair, what)


# ---- layer norm
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 512), (3, 130), (33, 128), (1000, 128), (257, 264), (7, 1024), (65, 1500), (9, 2048), (20, 4096),
                                    (6, 8192), (5, 8193), (3, 16384), (2, 20001), (5000, 72)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_layer_norm(tt, rows, n, dtype, pad, shift):
    gen = torch.Generator().manual_seed(rows + n)
    x, g = (randn(gen, rows, n, std=2) + randn(gen, rows, 1)).to(dtype), randn(gen, rows, n, dtype=dtype)
    w, b = randn(gen, n, dtype=dtype), randn(gen, n, dtype=dtype)
    want = ref.norm64(x, w, b, 1e-5, g)
    dx, dw, db = put(x, pad, shift).requires_grad_(), put(w, 0, shift).requires_grad_(), put(b, 0, shift).requires_grad_()
    y = tt.tt_layer_norm(dx, dw, db)
    check(y, want["out"], "out")
    grads = torch.autograd.grad(y, [dx, dw, db], put(g, pad, shift))
    for got, name in zip(grads, ("dx", "dweight", "dbias")):
        check(got, want[name], name)
    out = torch.full((rows, n + 3), 7.0, dtype=dtype, device="cuda")
    tt.tt_layer_norm_forward(dx, dw, db, out=out[:, :n])
    assert torch.equal(out[:, :n], y) and bool((out[:, n:] == 7).all())
    again = torch.autograd.grad(tt.tt_layer_norm(dx, dw, db), [dx, dw, db], put(g, pad, shift))
    assert all(torch.equal(p, q) for p, q in zip(grads, again))


@pytest.mark.parametrize("n,dtype", [(2, F32), (8, F32), (100, F32), (40, BF16), (200, BF16), (300, F32), (1000, F32), (3000, F32), (5000, BF16), (6000, F32), (9000, F32), (17000, BF16)])
def test_layer_norm_of_any_size(tt, n, dtype):
    """The norm and its gradients of rows near either end of the range, each between ordinary rows, which have the bits that they have alone."""
    gen = torch.Generator().manual_seed(n)
    w, b, grad, plain = randn(gen, n, dtype=dtype), randn(gen, n, dtype=dtype), randn(gen, 3, n, dtype=dtype), randn(gen, 2, n, dtype=dtype)

    def run(x, grad, eps):
        leaves = [put(t).requires_grad_() for t in (x, w, b)]
        y = tt.tt_layer_norm(*leaves, eps=eps)
        return [t.detach().cpu() for t in (y, *torch.autograd.grad(y, leaves, put(grad)))]
    for name, row, eps in far_rows(n, gen):
        eps = float(torch.tensor(eps, dtype=F32))
        x = torch.stack([plain[0], row.to(dtype), plain[1]])
        out, dx, dw, _ = run(x, grad, eps)
        want = ref.norm64(x, w, b, eps, grad)
        ref.check(out, *want["out"], name + " out")
        d = x.double() - x.double().mean(1, keepdim=True)
        rstd = 1 / ((d * d).mean(1, keepdim=True) + eps).sqrt()
        ref.check(dx, want["dx"][0], want["dx"][1] + stats_loss(want["dx"][0], rstd), name + " dx")
        ref.check(dw, want["dweight"][0], want["dweight"][1] + stats_loss((grad.double() * d * rstd).abs().sum(0), rstd.min()), name + " dweight")
        alone = run(x[:1], grad[:1], eps)
        assert torch.equal(out[0], alone[0][0]) and torch.equal(dx[0], alone[1][0]), name
    for value in (1e38, -3.3e38, 1e20, 1e-30):
        for eps in (1e-5, 1e-20, 1e-38):
            out, _, dw, _ = run(torch.full((2, n), value).to(dtype), grad[:2], eps)
            assert torch.equal(out, b.expand(2, n)) and not dw.any(), (value, eps)


def test_layer_norm_many_rows(tt):
    """More rows than workgroups take at a time; the sums over rows against 64 bits."""
    x = torch.randn(100003, 40, device="cuda")
    g = torch.randn_like(x)
    w = torch.randn(40, device="cuda").requires_grad_()
    y = tt.tt_layer_norm(x, w)
    (dw,) = torch.autograd.grad(y, w, g)
    want = ref.norm64(x.cpu(), w.detach().cpu(), grad=g.cpu())
    check(y, want["out"], "out")
    check(dw, want["dweight"], "dweight")


def test_layer_norm_of_more_dimensions_and_views(tt):
    x = torch.randn(4, 6, 16, device="cuda").transpose(0, 1).requires_grad_()
    y = tt.tt_layer_norm(x)
    assert y.shape == x.shape
    want = ref.norm64(x.detach().cpu().reshape(-1, 16), grad=torch.ones(24, 16))
    check(y.reshape(-1, 16), want["out"], "out")
    y.sum().backward()  # an expanded gradient
    check(x.grad.reshape(-1, 16), want["dx"], "dx")
    assert tt.tt_layer_norm(torch.randn(5, device="cuda")).shape == (5,)
    assert tt.tt_layer_norm(torch.empty(0, 8, device="cuda")).shape == (0, 8)


def differences(f, leaves, grads, eps=1e-3):
    """Directional derivatives of f (a float64 scalar of float32 leaves) by central differences, in random directions."""
    for leaf, grad in zip(leaves, grads):
        d = torch.randn_like(leaf)
        with torch.no_grad():
            was = leaf.clone()
            leaf.copy_(was + eps * d)
            up = f()
            leaf.copy_(was - eps * d)
            down = f()
            leaf.copy_(was)
        yield float((up - down) / (2 * eps)), float((grad.double() * d.double()).sum()), float((grad.double() * d.double()).abs().sum())


def test_gradients_by_differences(tt):
    """fp32 values are good to about 1e-6 of their size, so differences over 2e-3 to about 1e-3 of a sum's terms, and the third derivative adds
    eps^2: a hundredth of the sum of the terms' sizes is allowed."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w, b, r = f(12, 24).requires_grad_(), f(24).requires_grad_(), f(24).requires_grad_(), f(12, 24)
    norm = lambda: (tt.tt_layer_norm(x, w, b).double() * r).sum()
    for got, want, size in differences(norm, [x, w, b], torch.autograd.grad(norm(), [x, w, b])):
        assert abs(got - want) < 0.01 * size
    z, g = (4 * f(10, 8)).requires_grad_(), f(10, 3)
    for scores in ("softmax", "sigmoid"):
        for renorm in (True, False):
            route = lambda: (tt.tt_route(z, 3, scores=scores, renormalize=renorm).weights.double() * g).sum()
            for got, want, size in differences(route, [z], torch.autograd.grad(route(), [z])):
                assert abs(got - want) < 0.01 * size
    x, w, b = f(10, 16).requires_grad_(), f(50, 16).requires_grad_(), f(50).requires_grad_()
    labels = torch.randint(0, 50, (10,), device="cuda", generator=gen)
    loss = lambda: tt.tt_cross_entropy(x, w, labels, b).double()
    for got, want, size in differences(loss, [x, w, b], torch.autograd.grad(loss(), [x, w, b]), eps=1e-2):
        assert abs(got - want) < 0.01 * size


# ---- routing
@pytest.mark.parametrize("rows,num,k,dtype,scores,biased,groups,top,renorm,scale,pad", ROUTES + [
    (500, 64, 2, F32, "softmax", False, 1, 1, True, 1.0, 0), (301, 256, 8, F32, "sigmoid", True, 8, 4, True, 2.5, 8), (700, 160, 6, BF16, "softmax", True, 8, 3, False, 16.0, 0),
    (300, 512, 8, F16, "sigmoid", True, 16, 5, True, 1.0, 0)])
def test_route(tt, rows, num, k, dtype, scores, biased, groups, top, renorm, scale, pad):
    gen = torch.Generator().manual_seed(num + rows)
    z = routed(gen, rows, num, dtype)
    bias = torch.randint(-50, 51, (num,), generator=gen).float() * 1e-3 if biased else None
    if biased and num > 8:
        bias[4] = -math.inf
    how = dict(scores=scores, renormalize=renorm, scale=scale)
    want_w, want_e = ref.route64(z, k, bias, groups=groups, top_groups=top, **how)
    dz = put(z, pad).requires_grad_()
    r = tt.tt_route(dz, k, bias=put(bias), groups=groups, top_groups=top, **how)
    assert torch.equal(r.experts.cpu(), want_e)
    check(r.weights, (want_w, ref.weights_tol(want_w)), "weights")
    for got, want in zip(r[2:], ref.order_ref(want_e, num)):
        assert torch.equal(got.cpu(), want)
    g = randn(gen, rows, k)
    (grad,) = torch.autograd.grad(r.weights, dz, g.cuda())
    check(grad, ref.route_backward64(z, want_e, g, **how), "dlogits")


@pytest.mark.parametrize("logits,bias,scores", FAR_ROUTES)
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("num,dtype", [(4, F32), (64, F16), (300, F32)])
def test_route_of_scores_outside_single_precision(tt, logits, bias, scores, renorm, num, dtype):
    """Where the chosen scores are too small for fp32, weights and gradients are those of 64 bits; the rest of the experts is masked."""
    at = torch.arange(4) * (num // 4)
    z, b = torch.full((5, num), -math.inf), torch.zeros(num)
    z[:, at] = torch.tensor(logits)
    b[at] = torch.tensor(bias or [0.0] * 4)
    g = randn(torch.Generator().manual_seed(num), 5, 2)
    leaf = put(z.to(dtype)).requires_grad_()
    how = dict(scores=scores, renormalize=renorm, scale=2.5)
    r = tt.tt_route(leaf, 2, bias=put(b), **how)
    want_w, want_e = ref.route64(z.to(dtype), 2, b, **how)
    assert torch.equal(r.experts.cpu(), want_e)
    check(r.weights, (want_w, ref.weights_tol(want_w)), "weights")
    (dz,) = torch.autograd.grad(r.weights, leaf, g.cuda())
    check(dz, ref.route_backward_wide64(z.to(dtype), want_e, g, **how), "dlogits")


def test_close_scores_are_told_apart(tt):
    """Scores whose order single precision cannot tell: the larger logit wins by one unit in its last place, whatever the bias' size."""
    rows, num = 64, 40
    gen = torch.Generator().manual_seed(1)
    z = torch.randn(rows, 1, generator=gen).expand(rows, num).clone()
    best = torch.randint(0, num, (rows,), generator=gen)
    at = torch.arange(rows)
    z[at, best] = torch.nextafter(z[at, best], torch.full((rows,), 9.0))
    for scores in ("softmax", "sigmoid"):
        r = tt.tt_route(z.cuda(), 2, bias=torch.full((num,), 0.25, device="cuda"), scores=scores)
        assert torch.equal(r.experts[:, 0].cpu(), best)
        assert torch.equal(r.experts[:, 1].cpu(), torch.where(best == 0, 1, 0))


@pytest.mark.parametrize("rows,k,num", [(0, 2, 5), (1, 1, 1), (8192, 1, 64), (8193, 1, 64), (5000, 8, 256), (70001, 2, 1000), (40000, 3, 7)])
def test_expert_order(tt, rows, k, num):
    e = torch.randint(-1, num, (rows, k), generator=torch.Generator().manual_seed(rows))
    if rows > 100:
        e[7] = 2 ** 40
        e[: rows // 2] = torch.where(e[: rows // 2] >= 0, num - 1, -1)  # crowded
    got = tt.tt_expert_order(e.cuda(), num)
    for g, want in zip(got, ref.order_ref(e, num)):
        assert torch.equal(g.cpu(), want)


# ---- the experts' rows
@pytest.mark.parametrize("rows,k,num,n", [(1, 1, 1, 1), (1, 2, 64, 512), (48, 2, 64, 1024), (300, 3, 26, 130), (33, 8, 16, 2047), (5, 4, 9, 5000), (2000, 4, 64, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_expert_rows_and_combine(tt, rows, k, num, n, dtype, pad, shift):
    gen = torch.Generator().manual_seed(rows + n)
    e = torch.randint(-1, num, (rows, k), generator=gen)
    offsets, slots, sources = ref.order_ref(e, num)
    x, y, res, g, gxs = (randn(gen, r, n, dtype=dtype) for r in (rows, rows * k, rows, rows, rows * k))
    w, some = torch.rand(rows, k, generator=gen), sources >= 0
    y[~some] = math.nan
    gxs[~some] = math.nan
    leaves = [put(t, pad, shift).requires_grad_() for t in (x, y, res)] + [put(w).requires_grad_()]
    r = tt.Routes(leaves[3], *(t.cuda() for t in (e, offsets, slots, sources)))
    xs = tt.tt_expert_rows(leaves[0], r)
    assert torch.equal(xs.detach().cpu()[some], ref.rows_ref(x, slots)[some]) and not xs.detach().cpu()[~some].any()
    out = tt.tt_expert_combine(leaves[1], r, leaves[2])
    want = ref.combine64(y, slots, w, res, g)
    check(out, want["out"], "out")
    dx, dy, dres, dw = torch.autograd.grad([xs, out], leaves, [put(gxs, pad, shift), put(g, pad, shift)])
    check(dx, ref.combine64(gxs, slots)["out"], "dx")
    ref.check(dy.cpu()[some], want["dy"][0][some], want["dy"][1][some], "dy")
    assert not dy.cpu()[~some].any() and torch.equal(dres.cpu(), g)
    check(dw, want["dweights"], "dweights")
    left = torch.full((rows * k, n), 3.0, dtype=dtype, device="cuda")
    from paper_2507_14668_amd import binding
    binding.tt_expert_rows(leaves[0], r.slots, r.sources, out=left)
    assert bool((left.cpu()[~some] == 3).all()) and torch.equal(left.cpu()[some], xs.detach().cpu()[some])


# ---- the loss
BIG = [(1, 128, 1000, F32, True, "mean", 0, 0, 0), (300, 128, 2000, F32, True, "mean", 7, 0, 0), (257, 64, 5001, BF16, True, "none", 30, 0, 0),
       (513, 128, 20001, BF16, True, "mean", 50, 0, 0), (500, 136, 4099, F16, False, "none", 3, 8, 0), (700, 479, 1501, BF16, True, "sum", 1, 0, 1),
       (2048, 256, 6000, BF16, False, "mean", 200, 0, 0), (1500, 72, 9001, F16, True, "mean", 0, 0, 0), (2, 1024, 3000, BF16, True, "mean", 0, 0, 0),
       (9001, 16, 40, F32, True, "none", 4000, 0, 0), (3000, 128, 5001, F32, False, "mean", 11, 0, 0), (700, 256, 9000, F32, True, "mean", 5, 0, 0),
       (200, 520, 3001, F16, True, "sum", 9, 0, 0)]


@pytest.mark.parametrize("rows,dim,classes,dtype,biased,reduction,ignored,pad,shift", LOSSES + BIG)
def test_cross_entropy(tt, rows, dim, classes, dtype, biased, reduction, ignored, pad, shift):
    gen = torch.Generator().manual_seed(rows + classes)
    x, w = randn(gen, rows, dim, dtype=dtype), randn(gen, classes, dim, std=2 * dim ** -0.5, dtype=dtype)
    b = randn(gen, classes, dtype=dtype) if biased else None
    if biased and classes > 8:
        b[3] = -math.inf
    labels = torch.randint(0, classes, (rows,), generator=gen)
    labels[labels == 3] = 0
    skip = torch.randperm(rows, generator=gen)[:ignored]
    labels[skip] = -7
    x[skip] = math.nan
    grad = randn(gen, rows) if reduction == "none" else torch.tensor(1.0 if dtype != F16 else 300.0)
    leaves = [put(x, pad, shift), put(w, 0, shift)] + ([put(b, 0, shift)] if biased else [])
    call = lambda: tt.tt_cross_entropy(leaves[0], leaves[1], labels.cuda(), leaves[2] if biased else None, -7, reduction)
    evaluated = call()
    for t in leaves:
        t.requires_grad_()
    loss = call()
    assert torch.equal(loss, evaluated) and loss.dtype == F32
    grads = torch.autograd.grad(loss, leaves, grad.cuda())
    if rows == 0:
        assert loss == 0 and not grads[1].any()
        return
    want = ref.loss64(torch.where(torch.isnan(x), torch.zeros_like(x), x), w, labels, b, -7, reduction, grad)
    check(loss, want["loss"], "loss")
    for got, name in zip(grads, ("dx", "dw", "dbias")):
        check(got, want[name], name)
    assert not grads[0][skip.cuda()].any()
    again = torch.autograd.grad(call(), leaves, grad.cuda())
    assert all(torch.equal(p, q) for p, q in zip(grads, again))


@pytest.mark.parametrize("dim", [64, 100, 200])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gradients_of_nearly_sure_rows(tt, dim, dtype):
    """Rows whose label has almost all of the probability: what is left of the one after the label's share is formed before anything is rounded to 16
    bits, so the gradients keep their relative precision.  In the 2-norm: G and the result are rounded by half of eps each (three halves of
    it, twice over).  A logit of about 14 is off by at most 2 (dim + 2) u times the sum of its terms' sizes, which is itself here, and two of
    them make a probability.  The label's share comes of a sum near one and its logarithm, eight half units beside the 1 - p that is left."""
    gen = torch.Generator().manual_seed(dim)
    w = randn(gen, 500, dim, std=dim ** -0.5, dtype=dtype)
    labels = torch.randint(0, 500, (200,), generator=gen)
    x = (w[labels].double() / w[labels].double().norm(dim=1, keepdim=True) ** 2 * 13).to(dtype)  # the label's logit about 13, others of deviation 1
    grad = torch.tensor(1.0 if dtype != F16 else 200.0)
    want = ref.loss64(x, w, labels, grad=grad)
    p = float(torch.exp(-want["loss"][0]))
    assert 0.9 < p < 1
    leaves = [put(x).requires_grad_(), put(w).requires_grad_()]
    loss = tt.tt_cross_entropy(leaves[0], leaves[1], labels.cuda())
    check(loss, want["loss"], "loss")
    for got, name in zip(torch.autograd.grad(loss, leaves, grad.cuda()), ("dx", "dw")):
        check(got, want[name], name)
        off = (got.double().cpu() - want[name][0]).norm() / want[name][0].norm()
        assert off < 3 * torch.finfo(dtype).eps + 4 * (dim + 2) * ref.U * 14 + 8 * ref.U / (1 - p), (name, float(off))


@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (50, F16), (100, BF16), (128, F32), (136, BF16), (200, F32)])
@pytest.mark.parametrize("biased", [False, True])
def test_cross_entropy_of_large_logits(tt, size, dim, dtype, biased):
    """Finite logits of any size, far apart: losses to fp32's precision and never below zero, gradients of zeros and ones."""
    if dtype == F16:
        size = min(size, 2.0 ** 24 if not biased else 2.0 ** 14)
    x, w, b, labels = large_logits(size, dim, dtype, biased)
    grad = torch.tensor([1.0, -2.0, 0.5, 1.0, 2.0, 1.0, 0.25])
    want = large_logits64(x, w, b, labels, grad)
    leaves = [put(t).requires_grad_() for t in (x, w, b) if t is not None]
    loss = tt.tt_cross_entropy(leaves[0], leaves[1], labels.cuda(), leaves[2] if biased else None, reduction="none")
    assert bool((loss >= 0).all())
    check(loss, want["loss"], "loss")
    beyond = 2.0 ** 16 if dtype == F16 else math.inf  # (what rounds to fp16's infinity)
    for got, name in zip(torch.autograd.grad(loss, leaves, grad.cuda()), ("dx", "dw", "dbias")):
        ref.check(got.cpu().float().clamp(-beyond, beyond), want[name][0] if name != "dbias" else want[name][0][:, 0],
                  want[name][1] if name != "dbias" else want[name][1][:, 0], name)


@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (80, F16), (128, F32), (128, BF16), (136, F32), (136, BF16), (200, F16)])
def test_cross_entropy_of_sure_rows(tt, dim, dtype):
    """Row by row: the losses and gradients of rows that are nearly sure of their label keep their relative precision, however small they are."""
    x, w, labels = sure_rows(dim, dtype, 50)
    loss64, eloss, G, eG = sure_rows64(x, w, labels)
    if dtype != F32:
        eG = eG + 2.01 * torch.finfo(dtype).eps / 2 * G.abs() + (2.0 ** -37 if dtype == F16 else 2.0 ** -133)
    leaf = put(x).requires_grad_()
    loss = tt.tt_cross_entropy(leaf, put(w), labels.cuda(), reduction="none")
    check(loss, (loss64, eloss), "loss")
    (dx,) = torch.autograd.grad(loss, leaf, torch.ones_like(loss))
    check(dx[:, :64], (G, eG + ref.rounding(G, dtype)), "dx")
    assert not dx[:, 64:].any()


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("dim,dtype", [(64, F32), (64, BF16), (100, BF16), (128, F32), (136, BF16), (200, F32)])
def test_cross_entropy_of_large_operands(tt, dim, dtype, reduction):
    """Rows, then classes, near the type's largest number, and logits of ordinary size: gradients that the type holds are not lost on the way."""
    size, up, classes = 2.0 ** 125, 2.0 ** -125, 9
    for first, second in ((size, up), (up, size)):
        x, w = torch.zeros(3, dim), torch.zeros(classes, dim)
        x[0, 1], x[1, 1], x[2, 20] = first, -first, first / 2
        w[2, 1], w[3, 1], w[4, 20] = 2 * second, -second, second / 2
        labels, grad = torch.tensor([2, 3, 4]), torch.ones(3) if reduction == "none" else torch.tensor(1.0)
        x, w = x.to(dtype), w.to(dtype)
        want = ref.loss64(x, w, labels, reduction=reduction, grad=grad)
        leaves = [put(x).requires_grad_(), put(w).requires_grad_()]
        loss = tt.tt_cross_entropy(*leaves, labels.cuda(), reduction=reduction)
        check(loss, want["loss"], "loss")
        small = 2.0 ** -100 if dtype == F32 else 0.0  # (short fp32 rows: numbers below 2^-100 may have fewer bits)
        for got, name in zip(torch.autograd.grad(loss, leaves, grad.cuda()), ("dx", "dw")):
            check(got, (want[name][0], want[name][1] + small), name)


def test_routed_weights_changed_in_place(tt):
    z = torch.randn(50, 8, device="cuda", requires_grad=True)
    r = tt.tt_route(z, 2)
    plain, g = r.weights.detach().clone(), torch.randn(50, 2, device="cuda")
    (want,) = torch.autograd.grad(tt.tt_route(z, 2).weights, z, 2 * g)
    r.weights.mul_(2)
    assert torch.equal(r.weights, 2 * plain)
    (got,) = torch.autograd.grad(r.weights, z, g)
    assert torch.equal(got, want)


def test_no_rows(tt):
    """An empty batch through all of them, with gradients."""
    m = tt.TTExperts(16, 24, 8, 2)
    head = tt.TTSoftmaxLoss(16, 50, bias=True)
    x = torch.empty(0, 16, device="cuda").requires_grad_()
    loss = head(m(x), torch.empty(0, dtype=torch.int64, device="cuda"))
    loss.backward()
    assert loss == 0 and x.grad.shape == (0, 16)
    assert all(p.grad is not None and not p.grad.any() for p in list(m.parameters()) + list(head.parameters()))


def test_cross_entropy_of_frozen_parts(tt):
    """Each leaf alone gets what it gets beside the others."""
    gen = torch.Generator().manual_seed(3)
    x, w, b = randn(gen, 300, 64, dtype=BF16).cuda(), randn(gen, 1000, 64, dtype=BF16).cuda(), randn(gen, 1000, dtype=BF16).cuda()
    labels = torch.randint(0, 1000, (300,), generator=gen).cuda()
    together = None
    for pick in ((0, 1, 2), (0,), (1,), (0, 2)):
        leaves = [t.clone().requires_grad_(i in pick) for i, t in enumerate((x, w, b))]
        grads = torch.autograd.grad(tt.tt_cross_entropy(leaves[0], leaves[1], labels, leaves[2]), [leaves[i] for i in pick])
        together = together or grads
        for i, g in zip(pick, grads):
            assert torch.equal(g, together[i])


# ---- together
def layer64(m, x, mask):
    """TTExperts in 64 bits with autograd, from its parameters."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in m.named_parameters()}
    x = x.detach().double().cpu().requires_grad_()
    h = x
    if m.norm is not None:
        h = (x - x.mean(1, keepdim=True)) / (x.var(1, correction=0, keepdim=True) + m.norm.eps).sqrt() * p["norm.weight"] + p["norm.bias"]
    logits = h @ p["router.weight"].t()
    if mask is not None:
        logits = logits.masked_fill(~mask.cpu()[:, None], -math.inf)
    s = torch.sigmoid(logits) if m.route["scores"] == "sigmoid" else torch.softmax(logits, 1).nan_to_num(0.0)
    how = dict(m.route)
    renorm, scale = how.pop("renormalize"), how.pop("scale")
    _, e = ref.route64(logits.detach(), m.choices, None if m.balance is None else m.balance.cpu(), **how)
    there = e >= 0
    pick = torch.gather(s, 1, e.clamp(min=0)) * there
    w = scale * (pick / pick.sum(1, keepdim=True).clamp(min=1e-300) if renorm else pick)
    out = x if m.residual else torch.zeros_like(x)
    for j in range(m.choices):
        for r in range(x.shape[0]):
            if there[r, j]:
                k = e[r, j]
                z = h[r] @ p["up.weight"][k].t() + p["up.bias"][k]
                y = (z * torch.sigmoid(z)) @ p["down.weight"][k].t() + p["down.bias"][k]
                out = out + torch.zeros_like(x).index_put((torch.tensor([r]),), (w[r, j] * y)[None])
    return out, x, p


@pytest.mark.parametrize("how", [dict(), dict(scores="sigmoid", groups=4, top_groups=2, balance=True, scale=2.0), dict(norm=False, residual=False, renormalize=False)])
def test_experts_layer(tt, how):
    """norm, router, choice, the experts' products and the way back, with all gradients.  fp32 throughout: each of the seven steps is good to
    about 1e-6 of the largest of its terms, and steps pass errors on by factors of a few (the norm of the small matrices): 1e-4 of the
    largest value is allowed."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    m = tt.TTExperts(24, 40, 8, 3, generator=gen, **how)
    if m.balance is not None:
        m.balance.copy_(0.05 * torch.randn(8, device="cuda", generator=gen))
    x = torch.randn(37, 24, device="cuda", generator=gen).requires_grad_()
    mask = torch.rand(37, device="cuda", generator=gen) > 0.2
    g = torch.randn(37, 24, device="cuda", generator=gen)
    y = m(x, mask)
    y.backward(g)
    want, x64, p = layer64(m, x, mask)
    want.backward(g.double().cpu())
    near = lambda a, b: float((a.detach().cpu().double() - b).abs().max()) <= 1e-4 * float(b.abs().max() + 1e-3)
    assert near(y, want.detach()) and near(x.grad, x64.grad)
    for name, v in m.named_parameters():
        assert near(v.grad, p[name].grad), name
    if not m.residual:
        assert not y[~mask].any()


@pytest.mark.parametrize("n", [3, 128, 1000, 4096, 20000])
def test_layer_norm_of_equal_values(tt, n):
    """The bias, whatever eps is above zero and however far from zero the row is; no gradient of the row reaches the weight."""
    x = torch.tensor([1000.1, -0.1, 0.0, 77777.7], device="cuda")[:, None].expand(4, n).contiguous().requires_grad_()
    w, b = torch.full((n,), 3.0, device="cuda", requires_grad=True), torch.randn(n, device="cuda")
    y = tt.tt_layer_norm(x, w, b, eps=1e-12)
    assert torch.equal(y, b.expand(4, n))
    (dw,) = torch.autograd.grad(y.sum(), w)
    assert not dw.any()


def test_experts_layer_whatever_masked_rows_hold(tt):
    """NaN and infinities in masked rows: what the other rows get, and all gradients, have the bits that zeros there give."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    m = tt.TTExperts(48, 40, 8, 2, generator=gen, residual=False, dtype=torch.bfloat16)
    x = torch.randn(70, 48, device="cuda", generator=gen).bfloat16()
    mask = torch.rand(70, device="cuda", generator=gen) > 0.3
    runs = []
    for fill in (0.0, math.nan, math.inf):
        x[~mask] = fill
        leaf = x.clone().requires_grad_()
        y = m(leaf, mask)
        runs.append([y.detach(), *torch.autograd.grad(y.float().square().sum(), [leaf, *m.parameters()])])
        assert all(torch.equal(a, b) for a, b in zip(runs[0], runs[-1]))
    assert not runs[0][0][~mask].any() and not runs[0][1][~mask].any() and all(bool(t.isfinite().all()) for t in runs[0])


def test_a_model_of_them_learns_in_the_right_direction(tt):
    """Bags, experts and the loss, one step of each kind of optimizer: runs, and every parameter gets a gradient."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    bag = tt.TTEmbeddingBag(1000, 32, n=(10, 10, 10), d=(2, 4, 4), ranks=(8, 8), projection=48)
    experts = tt.TTExperts(48, 64, 4, 2, generator=gen)
    head = tt.TTSoftmaxLoss(48, 500, bias=True, generator=gen)
    model = torch.nn.ModuleList([bag, experts, head])
    opt = tt.TTOrthoSGD(model, lr=0.02)
    idx = torch.randint(0, 1000, (64, 5), device="cuda", generator=gen)
    labels = torch.randint(0, 500, (64,), device="cuda", generator=gen)
    loss = head(experts(bag(idx)), labels)
    loss.backward()
    assert all(p.grad is not None and bool(p.grad.isfinite().all()) for p in model.parameters())
    opt.step()
    assert bool(head(experts(bag(idx)), labels).isfinite())


# ---- streams, devices, graphs
def test_another_stream(tt):
    """Work on a given stream waits for what that stream waits for, and its memory is that stream's."""
    side = torch.cuda.Stream()
    x, w = torch.randn(300, 96, device="cuda"), torch.randn(700, 96, device="cuda")
    labels = torch.randint(0, 700, (300,), device="cuda")
    z = torch.randn(300, 64, device="cuda")
    stats = torch.empty(300, 2, device="cuda")
    want = [tt.tt_layer_norm_forward(x, stats=stats), *tt.tt_layer_norm_backward(x, None, stats, x, (True, True, True)), *tt.tt_cross_entropy_forward(x, w, labels),
            *tt.tt_route_forward(z, 4)]
    side.wait_stream(torch.cuda.current_stream())
    got = [tt.tt_layer_norm_forward(x, stats=stats, stream=side), *tt.tt_layer_norm_backward(x, None, stats, x, (True, True, True), stream=side),
           *tt.tt_cross_entropy_forward(x, w, labels, stream=side), *tt.tt_route_forward(z, 4, stream=side)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.cuda.stream(side):
        loss = tt.tt_cross_entropy(x.clone().requires_grad_(), w, labels)
        loss.backward()
    side.synchronize()
    assert torch.equal(loss.detach(), want[4])


def test_captured_and_replayed(tt):
    """A step of norm, routing, experts and loss with its gradients in a graph: each replay, with eager work in between, gives what the eager call
    gives on the same data."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    m = tt.TTExperts(64, 96, 16, 2, generator=gen, balance=True)
    head = torch.randn(3001, 64, device="cuda", generator=gen).requires_grad_()
    leaves = list(m.parameters()) + [head]
    x = torch.randn(200, 64, device="cuda", generator=gen)
    labels = torch.randint(0, 3001, (200,), device="cuda", generator=gen)

    def step():
        loss = tt.tt_cross_entropy(m(x), head, labels)
        return [loss.detach()] + list(torch.autograd.grad(loss, leaves))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        x.copy_(torch.randn(200, 64, device="cuda", generator=gen))
        labels.copy_(torch.randint(0, 3001, (200,), device="cuda", generator=gen))
        labels[:i] = -100
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_two_graphs_share_no_memory(tt):
    """Two captured losses replayed side by side on two streams, each with the workspace of its own capture."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    w = torch.randn(2000, 64, device="cuda", generator=gen)
    calls, graphs, outs = [], [], []
    for i in range(2):
        x = torch.randn(300, 64, device="cuda", generator=gen).requires_grad_()
        labels = torch.randint(0, 2000, (300,), device="cuda", generator=gen)
        calls.append((x, labels))
    run = lambda x, labels: torch.autograd.grad(tt.tt_cross_entropy(x, w, labels), x)[0]
    want = [run(*c) for c in calls]
    torch.cuda.synchronize()
    for c in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(*c))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals(tt):
    x, w = torch.randn(4, 8, device="cuda"), torch.randn(10, 8, device="cuda")
    labels, z = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.randn(4, 6, device="cuda")
    r = tt.tt_route(z, 2)
    with pytest.raises(TypeError):
        tt.tt_layer_norm(x.cpu())
    with pytest.raises(TypeError):
        tt.tt_layer_norm(x, torch.ones(8, dtype=BF16, device="cuda"))
    with pytest.raises(TypeError):
        tt.tt_layer_norm(x.double())
    with pytest.raises(ValueError):
        tt.tt_layer_norm(x, torch.ones(9, device="cuda"))
    with pytest.raises(tt.TTError):
        tt.tt_layer_norm(x, eps=-1.0)
    with pytest.raises(tt.TTError):
        tt.tt_layer_norm_forward(x, out=x)
    with pytest.raises(ValueError):
        tt.tt_route(z, 2, scores="tanh")
    for bad in (dict(k=7), dict(k=0), dict(k=2, groups=4), dict(k=2, groups=2, top_groups=3), dict(k=2, scale=math.nan), dict(k=4, groups=2, top_groups=1)):
        with pytest.raises(tt.TTError):
            tt.tt_route(z, **bad)
    with pytest.raises((TypeError, ValueError)):
        tt.tt_route(z, 2, bias=torch.zeros(5, device="cuda"))
    with pytest.raises(TypeError):
        tt.tt_route(z, 2, bias=torch.zeros(6, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        tt.tt_expert_rows(torch.randn(5, 8, device="cuda"), r)
    with pytest.raises(ValueError):
        tt.tt_expert_combine(torch.randn(4, 8, device="cuda"), r)
    with pytest.raises(TypeError):
        tt.tt_expert_combine(torch.randn(8, 8, device="cuda"), r, torch.randn(4, 8, dtype=F16, device="cuda"))
    with pytest.raises(ValueError):
        tt.tt_cross_entropy(x, w[:, :7], labels)
    with pytest.raises(TypeError):
        tt.tt_cross_entropy(x, w, labels.int())
    with pytest.raises(ValueError):
        tt.tt_cross_entropy(x, w, labels[:3])
    with pytest.raises(ValueError):
        tt.tt_cross_entropy(x, w, labels, reduction="max")
    with pytest.raises(TypeError):
        tt.tt_cross_entropy(x, w.bfloat16(), labels)
    with pytest.raises(tt.TTError):
        tt.tt_cross_entropy_forward(x, w, labels, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(tt.TTError):
        tt.tt_cross_entropy(x, w[:0], labels)
