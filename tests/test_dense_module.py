"""The dense layers' module side on the CPU: what reaches the library, what is refused, what an optimizer step computes.  The library's calls are
replaced by their plain forms."""
import copy

import pytest
import torch
import torch.autograd.forward_ad as fw

import dense_ref as ref


@pytest.fixture
def tt(monkeypatch):
    import paper_2507_14668_amd as tt
    from paper_2507_14668_amd import binding

    def forward(x, w, bias=None, residual=None, activation="none", offsets=None, out=None, pre=None, workspace=None, stream=None):
        y, _, z, _ = ref.forward64(x, w, bias, residual, activation, offsets)
        if pre is not None:
            pre.copy_(z)
        return y.to(x.dtype)

    def orthogonalize(g, steps=5, coefficients=binding.ORTHO_COEFFICIENTS, eps=1e-7, out=None, workspace=None, stream=None):
        assert g.stride(-1) == 1 and g.stride(-2) >= g.shape[-1]
        x = g.reshape((-1,) + g.shape[-2:])
        return ref.ortho(x, steps=steps, coefficients=coefficients, eps=eps).reshape(g.shape).to(g.dtype)
    monkeypatch.setattr(binding, "tt_dense_forward", forward)
    monkeypatch.setattr(binding, "tt_orthogonalize", orthogonalize)

    def core_update(table, dcores, momenta, lr, momentum=0.95, nesterov=True, steps=5, coefficients=binding.ORTHO_COEFFICIENTS, eps=1e-7, workspace=None,
                    stream=None):
        r, n, d = table.r, table.n, table.d
        for k, (c, g, m) in enumerate(zip(table.cores, dcores, momenta)):
            m.mul_(momentum).add_(g)
            u = (g + momentum * m if nesterov else m).view(r[k], n[k], d[k] * r[k + 1]).transpose(0, 1)
            u = u.reshape(n[k], d[0], r[1]) if k == 0 else u
            o = ref.ortho(u, steps=steps, coefficients=coefficients, eps=eps) * max(1.0, u.shape[1] / u.shape[2]) ** 0.5
            c.sub_((lr * o).float().reshape(n[k], r[k], -1).transpose(0, 1).reshape(-1))
    monkeypatch.setattr(binding, "tt_core_ortho_update", core_update)

    class Table:
        def __init__(self, num_rows, n, d, r, cores):
            self.n, self.d, self.r, self.cores = n, d, r, cores
    monkeypatch.setattr(binding, "Table", Table)
    return tt


def test_forward_mode_is_refused(tt):
    """A tangent is never dropped: frozen weights, no_grad and trainable weights alike."""
    x, w = torch.randn(3, 4), torch.randn(5, 4)
    with fw.dual_level():
        dual = fw.make_dual(x, torch.ones_like(x))
        for weight in (w, w.clone().requires_grad_(True)):
            for args in ((dual, weight), (x, weight, fw.make_dual(torch.zeros(5), torch.ones(5))), (x, weight, None, fw.make_dual(torch.zeros(3, 5), torch.ones(3, 5)))):
                with pytest.raises((RuntimeError, NotImplementedError)):
                    tt.tt_dense(*args)
                with torch.no_grad(), pytest.raises((RuntimeError, NotImplementedError)):
                    tt.tt_dense(*args)
        assert torch.allclose(tt.tt_dense(x, w), x @ w.t())  # no tangents: as ever
    assert torch.allclose(tt.tt_dense(x, w), x @ w.t())


def ortho_step64(p, g, m, lr, mu, matrix, eps):
    """One step in 64 bits: (new parameter, new momentum)."""
    m = mu * m.double() + g.double()
    u = g.double() + mu * m
    if matrix:
        u = max(1.0, p.shape[-2] / p.shape[-1]) ** 0.5 * ref.ortho(u.reshape((-1,) + u.shape[-2:]), eps=eps).reshape(u.shape)
    return p.double() - lr * u, m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("groups", [None, 3])
@pytest.mark.parametrize("scale", [1e-9, 1e-8, 1.0, 1e5])
def test_optimizer_steps_at_any_scale(tt, dtype, groups, scale):
    """Momenta far below and above the range of half precision: the step is that of 64 bits, rounded to the parameter's type once."""
    layer = tt.TTDense(24, 16, groups=groups, device="cpu", dtype=dtype, generator=torch.Generator().manual_seed(0))
    opt = tt.TTOrthoSGD(layer, lr=0.01, momentum=0.95, eps=0.0)
    gen = torch.Generator().manual_seed(1)
    for p in (layer.weight, layer.bias):
        opt.state[p]["momentum"] = torch.randn(p.shape, generator=gen) * scale
        p.grad = (torch.randn(p.shape, generator=gen) * min(scale, 1e3)).to(dtype)
    want = [ortho_step64(p.detach(), p.grad, opt.state[p]["momentum"], 0.01, 0.95, p is layer.weight, 0.0) for p in (layer.weight, layer.bias)]
    opt.step()
    for p, (new, m) in zip((layer.weight, layer.bias), want):
        assert bool(torch.isfinite(new.to(dtype)).all()) == bool(torch.isfinite(p).all())
        fine = torch.isfinite(new.to(dtype))
        # half a step of the type, and the step itself in fp32: its singular values are near one, and errors of 2^-23 of u are taken 485 times at most
        off = 485 * 2.0 ** -22 * 0.01 if p is layer.weight else 2.0 ** -21 * 0.01 * float(m.abs().max()) * 2
        ref.check(p.detach()[fine], new[fine], ref.rounding(new, dtype)[fine] + off, "parameter")
        ref.check(opt.state[p]["momentum"], m, 2.0 ** -22 * m.abs().max().expand(m.shape), "momentum")


def one_bag(tt, seed=0):
    bag = tt.TTEmbeddingBag(24, 16, n=(2, 3, 4), d=(2, 2, 4), ranks=(4, 3), device="cpu", generator=torch.Generator().manual_seed(seed))
    for c in bag.cores():
        c.grad = torch.randn(c.shape, generator=torch.Generator().manual_seed(9))
    return bag


@pytest.mark.parametrize("frozen", [(0,), (1,), (0, 2), (0, 1, 2)])
def test_frozen_cores_do_not_hold_up_the_others(tt, frozen):
    bag, other = one_bag(tt), one_bag(tt)
    for k in frozen:
        bag.cores()[k].requires_grad_(False)
        bag.cores()[k].grad = None
    for m in (bag, other):
        opt = tt.TTOrthoSGD(m, lr=0.01)
        opt.step()
        opt.step()
    start = one_bag(tt)
    for k in range(3):
        assert torch.equal(bag.cores()[k], (start if k in frozen else other).cores()[k])
        assert torch.equal(other.cores()[k], start.cores()[k]) is False


def test_shared_parameters_take_one_step(tt):
    class Model(torch.nn.Module):
        def __init__(self, shared):
            super().__init__()
            gen = torch.Generator().manual_seed(0)
            self.a, self.b = (tt.TTDense(12, 8, device="cpu", generator=gen) for _ in range(2))
            self.s, self.t = one_bag(tt, 1), one_bag(tt, 2)
            if shared:
                self.b.weight = self.a.weight
                self.t.core1 = self.s.core1
            for layer in (self.a, self.b):
                layer.weight.grad = torch.ones_like(layer.weight)
    models = [Model(True), Model(False)]
    for m in models:
        opt = tt.TTOrthoSGD(m, lr=0.01)
        for group in opt.param_groups:
            assert len({id(p) for p in group["params"]}) == len(group["params"])
        opt.step()
    both, apart = models
    assert torch.equal(both.a.weight, apart.a.weight) and both.b.weight is both.a.weight
    for k in range(3):
        assert torch.equal(both.s.cores()[k], apart.s.cores()[k])
        assert torch.equal(both.t.cores()[k], both.s.cores()[k] if k == 1 else apart.t.cores()[k])


@pytest.mark.parametrize("nesterov", [True, False])
def test_gradients_of_any_strides(tt, nesterov):
    """A gradient that a caller set, with its columns apart, gives the step of the same numbers in a row."""
    layers = [tt.TTDense(12, 8, groups=2, device="cpu", generator=torch.Generator().manual_seed(0)) for _ in range(2)]
    g = torch.randn(2, 8, 12, generator=torch.Generator().manual_seed(1))
    layers[0].weight.grad, layers[1].weight.grad = g, g.transpose(1, 2).contiguous().transpose(1, 2)
    for layer in layers:
        opt = tt.TTOrthoSGD(layer, lr=0.01, nesterov=nesterov)
        opt.step()
        opt.step()
    assert torch.equal(layers[0].weight, layers[1].weight)


def test_copies_of_model_and_optimizer(tt):
    bag = one_bag(tt)
    opt = tt.TTOrthoSGD(bag, lr=0.01)
    opt.step()
    bag2, opt2 = copy.deepcopy((bag, opt))
    for c, c2 in zip(bag.cores(), bag2.cores()):
        c2.grad = c.grad.clone()
    opt.step()
    opt2.step()
    assert all(torch.equal(a, b) and a is not b for a, b in zip(bag.cores(), bag2.cores()))


@pytest.mark.parametrize("x,w,groups", [((1, 2 ** 32 + 16), (8, 2 ** 32 + 16), 0), ((1, 8), (2 ** 32 + 16, 8), 0), ((4, 8), (2 ** 32 + 1, 1, 8), 2 ** 32 + 1),
                                        ((1, 2 ** 31 + 8), (4, 2 ** 31 + 8), 0)])
def test_sizes_past_32_bits_are_refused(tt, monkeypatch, x, w, groups):
    """Sizes go to the library in 32 bits: larger ones must not arrive there as what is left of them (tensors without memory)."""
    from paper_2507_14668_amd import binding
    monkeypatch.setattr(binding, "_index", lambda t, name, dtype, at: 0)
    make = lambda shape: torch.empty(shape, dtype=torch.bfloat16, device="meta")
    off = torch.empty(groups + 1, dtype=torch.int64, device="meta") if groups else None
    with pytest.raises(binding.TTError) as e:
        binding._dense_op(make(x), make(w), "none", off)
    assert e.value.status == binding.TT_ERR_SHAPE


def test_compression_ratio_is_the_cores(tt):
    make = lambda **kw: tt.TTEmbeddingBag(1000, 16, n=(10, 10, 10), d=(2, 2, 4), ranks=(4, 4), device="cpu", **kw)
    ratio = "%.1fx smaller than dense" % (1000 * 16 / (10 * 2 * 4 + 4 * 10 * 2 * 4 + 4 * 10 * 4))
    assert ratio in repr(make()) and ratio in repr(make(projection=512))


@pytest.mark.parametrize("projection", [None, 12])
def test_modules_pickled_without_a_projection(tt, projection):
    """A module whose pickle knows of no projection has none; others keep theirs."""
    fused = tt.TTFusedEmbeddingBags([(24, (2, 3, 4)), (6, (1, 2, 3))], 16, (2, 2, 4), (4, 3), device="cpu", projection=projection)
    bag = tt.TTEmbeddingBag(24, 16, n=(2, 3, 4), d=(2, 2, 4), ranks=(4, 3), device="cpu", projection=projection)
    for m in (bag, fused):
        state = dict(m.__dict__)
        if projection is None:
            del state["projection"]
        again = type(m).__new__(type(m))
        again.__setstate__(state)
        assert again.projection is m.projection
        assert torch.equal(copy.deepcopy(m).core0, m.core0)


def test_steps_are_checked_before_coefficients_are_laid_out(tt):
    """A number of steps that the library would refuse is refused before a list of that length is made."""
    import os
    import re
    from paper_2507_14668_amd import binding
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tt_emb.h")).read()
    assert binding.TT_ORTHO_MAX_STEPS == int(re.search(r"#define TT_ORTHO_MAX_STEPS (\d+)", header).group(1))
    assert len(binding._coefficients(32, (1, 2, 3))) == 96
    for steps in (0, -1, 33, 10 ** 6):
        with pytest.raises(ValueError):
            binding._coefficients(steps, (1, 2, 3))
