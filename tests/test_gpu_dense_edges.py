"""The dense operators on the GPU where a last bit, a special value or a second caller decides: relu's sign, numbers near the ends of the
range, NaN beside sums, gelu's tail, kept state."""
import math

import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tt():
    import paper_2507_14668_amd as tt
    return tt


def normal(*shape, seed=0, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


@pytest.mark.parametrize("rows,k,n,sizes", [(1, 128, 512, None), (48, 200, 96, None), (300, 128, 130, None), (300, 3000, 260, None), (4096, 128, 2048, None),
                                            (5000, 77, 1500, None), (3000, 96, 640, (1000, 0, 7, 1993))])
def test_relu_decides_the_sign_exactly(tt, rows, k, n, sizes):
    """Biases that cancel a column's sum for one row of the first group down to its last bits: the stored pre-activation has the exact value's sign,
    and the output and the gradients follow it."""
    groups = 0 if sizes is None else len(sizes)
    lead = (groups,) if groups else ()
    x, w, bias = normal(rows, k, seed=rows), normal(*lead, n, k, seed=k, std=k ** -0.5), normal(*lead, n, seed=n)
    off = None if sizes is None else torch.tensor([0] + list(sizes)).cumsum(0)
    cols = torch.arange(n)
    at = cols % (sizes[0] if groups else rows)
    w0, b0 = (w[0], bias[0]) if groups else (w, bias)
    terms = x[at].double() * w0.double()
    b0.copy_(-terms.sum(1).float())
    exact, noise = terms.sum(1) + b0.double(), 2 * k * 2.0 ** -53 * terms.abs().sum(1)
    dx, dw, db, doff = x.cuda(), w.cuda(), bias.cuda(), None if off is None else off.cuda()
    pre = torch.empty(rows, n, device="cuda")
    out = tt.tt_dense_forward(dx, dw, db, None, "relu", offsets=doff, pre=pre)
    got, value = pre.cpu()[at, cols].double(), out.cpu()[at, cols]
    assert bool(((got - exact).abs() <= ref.U * exact.abs() + noise).all())
    clear = exact.abs() > noise
    assert int(clear.sum()) > 0.5 * n and torch.equal((value > 0)[clear], (exact > 0)[clear])
    grad = torch.zeros(rows, n)
    grad[at, cols] = 1.0
    db = tt.tt_dense_backward(dx, dw, grad.cuda(), pre, "relu", offsets=doff, needs=(False, False, True))[2].cpu()
    assert torch.equal(((db[0] if groups else db) == 1)[clear], (exact > 0)[clear])
    assert torch.equal(tt.tt_dense_forward(dx, dw, db.cuda() * 0 + bias.cuda(), None, "relu", offsets=doff), out)


@pytest.mark.parametrize("seed", range(4))
def test_relu_gradients_of_a_large_batch(tt, seed):
    """16384 x 128 -> 512: every one of 8 million signs is that of 64 bits, and the gradients are the formula's to fp32 rounding."""
    rows, k, n = 16384, 128, 512
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, w, bias, grad = (torch.randn(*s, generator=gen, device="cuda") for s in ((rows, k), (n, k), (n,), (rows, n)))
    w, bias = w * k ** -0.5, bias * 0.1
    leaves = [t.requires_grad_(True) for t in (x, w, bias)]
    got = torch.autograd.grad(tt.tt_dense(x, w, bias, None, "relu"), leaves, grad)
    with torch.no_grad():
        z = x.double() @ w.double().t() + bias.double()
        dz = torch.where(z > 0, grad.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        want = (dz @ w.double(), dz.t() @ x.double(), dz.sum(0))
    for g, v, name in zip(got, want, ("dx", "dw", "dbias")):
        # one sign the other way moves a row of dx by about 5e-4 of the whole; sums of up to 16384 terms in fp32 are off by a few 1e-6 in 2-norm
        assert float((g.double() - v).norm() / v.norm()) < 2e-5, name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows,k,n,groups", [(520, 4096, 2560, 0), (5000, 1024, 1024, 12), (300, 256, 264, 0)])
def test_bias_gradient_beside_special_values(tt, rows, k, n, groups, dtype):
    """A NaN or an infinity in a column of the gradient reaches that column's sum only, whatever else is asked for (the first two sizes are those
    of the largest tiles, whole and cut along the rows)."""
    lead = (groups,) if groups else ()
    x, w, grad = normal(rows, k, dtype=dtype).cuda(), torch.zeros(*lead, n, k, dtype=dtype, device="cuda"), normal(rows, n, seed=1, dtype=dtype).cuda()
    off = None
    if groups:
        off = torch.tensor([0] + [rows - 8 * (groups - 1) + 8 * g for g in range(groups)], device="cuda")
    clean = tt.tt_dense_backward(x, w, grad, offsets=off)[2]
    for value, cols in ((math.nan, (7,)), (math.inf, (7, n - 1)), (-math.inf, (130,))):
        bad = grad.clone()
        bad[11, list(cols)] = value
        want = clean.clone()
        want[(0, list(cols)) if groups else list(cols)] = value
        for needs in ((False, True, True), (False, False, True)):
            got = tt.tt_dense_backward(x, w, bad, offsets=off, needs=needs)[2]
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(3.0, 4.0, 5.0), want.nan_to_num(3.0, 4.0, 5.0)), (value, cols, needs)


@pytest.mark.parametrize("small,large", [(2.0 ** -115, 2.0 ** 100), (1e-35, 1e20), (2e-38, 1e25), (1e-30, 1e-6), (2.0 ** -101, 1.0)])
@pytest.mark.parametrize("rows,k,n", [(8, 64, 96), (300, 256, 512), (2000, 96, 2100), (500, 4096, 130)])
def test_small_numbers_beside_large_ones(tt, rows, k, n, small, large):
    """Normal fp32 numbers near the lower end, all of an operand or one of each row, keep their 24 bits whatever they are multiplied by: within
    2 (K + 2) u sum |terms| (and half of the smallest number for each term), forward and backward."""
    x, w = normal(rows, k, seed=1).clamp(-3, 3), normal(n, k, seed=2).clamp(-3, 3)
    for a, b in ((small * x, large * w), (large * x, small * w)):
        for single in (False, True):
            if single:
                a, b = a.clone(), b.clone()
                t = a if small * 100 > float(a.abs().max()) else b
                keep = torch.zeros_like(t)
                keep[torch.arange(t.shape[0]), torch.arange(t.shape[0]) % k] = 1.0
                t.mul_(keep)
            got = tt.tt_dense_forward(a.cuda(), b.cuda()).cpu()
            bound = lambda k, size: 2 * (k + 2) * ref.U * size + (k + 1) * 2.0 ** -149
            ref.check(got, a.double() @ b.double().t(), bound(k, a.double().abs() @ b.double().abs().t()), "out")
            grad = b[:rows % n + 1, :1].expand(-1, rows).t().contiguous() if n > rows else b[:, :1].t().expand(rows, -1).contiguous()
            grad = grad[:, :n] if grad.shape[1] >= n else grad.repeat(1, -(-n // grad.shape[1]))[:, :n].contiguous()
            weight = a[:1].expand(n, -1).contiguous()
            dx, dw, _ = tt.tt_dense_backward(a.cuda(), weight.cuda(), grad.cuda())
            ref.check(dx.cpu(), grad.double() @ weight.double(), bound(n, grad.double().abs() @ weight.double().abs()), "dx")
            ref.check(dw.cpu(), grad.double().t() @ a.double(), bound(rows, grad.double().abs().t() @ a.double().abs()), "dw")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_gelu_of_16_bits_over_its_tail(tt, dtype):
    """Value and slope to half a step of the type, relative to themselves, down to where they leave its range."""
    z = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dtype)
    z = z[torch.isfinite(z) & (z >= -12.75) & (z <= 8) & (z.float().abs() >= 2.0 ** -8)]
    # Phi to 2e-6, the rounding of z^2 / 2 and of exp's argument, a few units for the rest; then half a step of the type
    z64 = z.double()
    phi, bell = 0.5 * torch.erfc(-z64 / math.sqrt(2)), torch.exp(-0.5 * z64 * z64) / math.sqrt(2 * math.pi)
    near = 2e-6 + (z64 * z64 + 8) * ref.U
    x, one = z[:, None].cuda(), torch.ones(1, 1, dtype=dtype, device="cuda")
    want = z64 * phi
    ref.check(tt.tt_dense_forward(x, one, activation="gelu").cpu()[:, 0], want, near * want.abs() + ref.rounding(want, dtype), "gelu")
    want = phi + z64 * bell
    got = tt.tt_dense_backward(x, one, torch.ones_like(x), x, "gelu", needs=(True, False, False))[0]
    ref.check(got.cpu()[:, 0], want, near * (phi + z64.abs() * bell) + ref.rounding(want, dtype), "slope")


@pytest.mark.parametrize("rows,k,n", [(8, 64, 96), (300, 256, 512), (60, 5000, 70), (2000, 96, 2100)])
def test_float32_overflows_to_infinity(tt, rows, k, n):
    """Positive terms only: a sum clearly past the range is an infinity (no NaN, no number), one clearly within it is a number."""
    x, w = normal(rows, k, seed=1).abs() + 0.1, normal(n, k, seed=2).abs() + 0.1
    size = x.double() @ w.double().t()
    x = x * float(3.4028e38 / size.median())  # half of the results are past the range
    want = x.double() @ w.double().t()
    for act in ("none", "relu"):
        got = tt.tt_dense_forward(x.cuda(), w.cuda(), activation=act).cpu()
        margin = 2 * (k + 2) * ref.U
        over, within = want > 3.4028236e38 * (1 + margin), want < 3.4028234e38 * (1 - margin)
        assert int(over.sum()) > rows * n // 4 and bool((got[over] == math.inf).all())
        ref.check(got[within], want[within], margin * want[within], act)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("groups", [None, 3])
@pytest.mark.parametrize("scale", [1e-9, 1.0, 1e5])
def test_optimizer_steps_at_any_scale(tt, dtype, groups, scale):
    """Momenta far below and above the range of half precision: the step is that of 64 bits, rounded to the parameter's type once."""
    layer = tt.TTDense(24, 16, groups=groups, dtype=dtype, generator=torch.Generator(device="cuda").manual_seed(0))
    opt = tt.TTOrthoSGD(layer, lr=0.01, momentum=0.95, eps=0.0)
    want = []
    for i, p in enumerate((layer.weight, layer.bias)):
        m, g = normal(*p.shape, seed=i, std=scale), normal(*p.shape, seed=9 + i, std=min(scale, 1e3)).to(dtype)
        opt.state[p]["momentum"], p.grad = m.cuda(), g.cuda()
        m64 = 0.95 * m.double() + g.double()
        u = g.double() + 0.95 * m64
        if p is layer.weight:
            u = ref.ortho(u.reshape((-1,) + u.shape[-2:]), eps=0.0).reshape(u.shape)
        want.append((p.detach().cpu().double() - 0.01 * u, m64))
    opt.step()
    for p, (new, m) in zip((layer.weight, layer.bias), want):
        fine = torch.isfinite(new.to(dtype))
        assert torch.equal(torch.isfinite(p.detach().cpu()), fine)
        # half a step of the type, and the step itself in fp32: its singular values are near one, and errors of 2^-22 of u are taken 485 times at most
        off = 485 * 2.0 ** -22 * 0.01 if p is layer.weight else 2.0 ** -21 * 0.01 * float(m.abs().max()) * 2
        ref.check(p.detach().cpu()[fine], new[fine], ref.rounding(new, dtype)[fine] + off, "parameter")
        ref.check(opt.state[p]["momentum"].cpu(), m, 2.0 ** -22 * m.abs().max().expand(m.shape), "momentum")


def test_frozen_core_on_the_gpu(tt):
    """A table whose middle core is frozen trains the other two as it would beside a trained one."""
    bags = [tt.TTEmbeddingBag(24, 16, n=(2, 3, 4), d=(2, 2, 4), ranks=(4, 3), generator=torch.Generator(device="cuda").manual_seed(0)) for _ in range(2)]
    bags[0].core1.requires_grad_(False)
    idx, off = torch.arange(24, device="cuda"), torch.arange(0, 24, 3, device="cuda")
    start = [c.detach().clone() for c in bags[0].cores()]
    for bag in bags:
        opt = tt.TTOrthoSGD(bag, lr=0.01)
        bag(idx, off).square().sum().backward()
        opt.step()
    assert bags[0].core1.grad is None and torch.equal(bags[0].core1, start[1]) and not torch.equal(bags[1].core1, start[1])
    for k in (0, 2):
        assert torch.equal(bags[0].cores()[k], bags[1].cores()[k]) and not torch.equal(bags[0].cores()[k], start[k])
