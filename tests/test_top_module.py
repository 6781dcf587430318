"""Layer norm, routing, the experts' rows and the softmax loss on the CPU: the structs' layout, what reaches the library, what is refused.  The
library's calls are replaced by their plain forms."""
import ctypes
import math
import os
import subprocess

import pytest
import torch
import torch.autograd.forward_ad as fw

import top_ref as ref
from test_abi import ROOT, _header_struct_fields


def test_struct_mirrors_match_header_layout(tmp_path):
    from paper_2507_14668_amd import binding
    pairs = (("tt_norm", binding.CNorm), ("tt_route", binding.CRoute), ("tt_deal", binding.CDeal), ("tt_loss", binding.CLoss), ("tt_dense", binding.CDense))
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "tt_emb.h"', "int main(void) {"]
    for name, _ in pairs:
        lines.append('printf("%s sizeof %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s %s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in _header_struct_fields(name)]
    lines.append("return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()}
    for name, cls in pairs:
        assert ctypes.sizeof(cls) == got[name, "sizeof"], name
        assert [f for f, _ in cls._fields_] == [f for f, _ in _header_struct_fields(name)], name
        for f, _ in cls._fields_:
            assert getattr(cls, f).offset == got[name, f], (name, f)


def test_limits_match_the_header():
    from paper_2507_14668_amd import binding
    text = open(os.path.join(ROOT, "include", "tt_emb.h")).read()
    for name in ("TT_ROUTE_MAX_EXPERTS", "TT_ROUTE_MAX_CHOICES", "TT_ROUTE_MAX_GROUPS"):
        assert "#define %s %d\n" % (name, getattr(binding, name)) in text


def rows_only(*ts):
    """As the library asks for them: columns next to each other, rows that do not overlap."""
    for t in ts:
        assert t is None or t.dim() != 2 or ((t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]))


@pytest.fixture
def tt(monkeypatch):
    import paper_2507_14668_amd as tt
    from paper_2507_14668_amd import binding
    import dense_ref

    def norm(x, weight=None, bias=None, eps=1e-5, out=None, stats=None, stream=None):
        rows_only(x)
        return ref.norm64(x, weight, bias, eps)["out"][0].to(x.dtype)

    def norm_back(x, weight, stats, grad_out, needs=(True,) * 3, workspace=None, stream=None):
        rows_only(x, grad_out)
        r = ref.norm64(x, weight, None, 1e-5, grad_out)
        return tuple(r[k][0].to(x.dtype) if n else None for k, n in zip(("dx", "dweight", "dbias"), needs))

    def route(logits, k, bias=None, scores="softmax", groups=1, top_groups=None, renormalize=False, scale=1.0, workspace=None, stream=None):
        rows_only(logits)
        w, e = ref.route64(logits, k, bias, scores, groups, top_groups, renormalize, scale)
        return (w.float(), e, *ref.order_ref(e, logits.shape[1]))

    def route_back(logits, experts, grad, scores="softmax", renormalize=False, scale=1.0, stream=None):
        assert grad.is_contiguous()
        return ref.route_backward64(logits, experts, grad, scores, renormalize, scale)[0].to(logits.dtype)

    def rows(x, slots, sources, out=None, stream=None):
        rows_only(x)
        return torch.nan_to_num(ref.rows_ref(x, slots), nan=0.0)

    def combine(y, slots, weights=None, residual=None, out=None, stream=None):
        rows_only(y, residual)
        return ref.combine64(y, slots, weights, residual)["out"][0].to(y.dtype)

    def combine_back(y, slots, sources, weights, grad, needs=(True, True), stream=None):
        rows_only(y, grad)
        r = ref.combine64(y, slots, weights, None, grad)
        return torch.nan_to_num(r["dy"][0], nan=0.0).to(y.dtype) if needs[0] else None, r["dweights"][0].float() if needs[1] else None

    def loss(x, w, labels, bias=None, ignore_index=-100, reduction="mean", workspace=None, stream=None):
        rows_only(x)
        assert w.is_contiguous() and labels.is_contiguous()
        return ref.loss64(x, w, labels, bias, ignore_index, reduction)["loss"][0].float(), torch.zeros(x.shape[0], 2)

    def loss_back(x, w, labels, stats, grad, bias=None, ignore_index=-100, reduction="mean", needs=(True,) * 3, workspace=None, stream=None):
        r = ref.loss64(x, w, labels, bias, ignore_index, reduction, grad)
        return tuple(r[k][0].to(x.dtype) if n else None for k, n in zip(("dx", "dw", "dbias"), needs))

    def dense(x, w, bias=None, residual=None, activation="none", offsets=None, out=None, pre=None, workspace=None, stream=None):
        y, _, z, _ = dense_ref.forward64(x, w, bias, residual, activation, offsets)
        if pre is not None:
            pre.copy_(torch.nan_to_num(z))
        return torch.nan_to_num(y).to(x.dtype)

    def dense_back(x, w, grad, pre=None, activation="none", offsets=None, needs=(True,) * 3, workspace=None, stream=None):
        d, _ = dense_ref.backward64(x, w, grad, pre, activation, offsets)
        return tuple(torch.nan_to_num(v).to(x.dtype) if n else None for v, n in zip(d, needs))
    for name, f in (("tt_layer_norm_forward", norm), ("tt_layer_norm_backward", norm_back), ("tt_route_order", route), ("tt_route_backward", route_back),
                    ("tt_expert_rows", rows), ("tt_expert_combine", combine), ("tt_expert_combine_backward", combine_back), ("tt_cross_entropy_forward", loss),
                    ("tt_cross_entropy_backward", loss_back), ("tt_dense_forward", dense), ("tt_dense_backward", dense_back)):
        monkeypatch.setattr(binding, name, f)
    return tt


def calls(tt):
    """Each operator as a function of one tensor."""
    labels, r = torch.tensor([0, 2, -100]), None
    w = torch.randn(4, 6)

    def routes():
        return tt.tt_route(torch.arange(12.0).view(3, 4), 2)
    return {
        "norm": lambda x: tt.tt_layer_norm(x),
        "route": lambda x: tt.tt_route(x, 2).weights,
        "rows": lambda x: tt.tt_expert_rows(x, routes()),
        "combine": lambda x: tt.tt_expert_combine(x.repeat(2, 1), routes(), x),
        "loss": lambda x: tt.tt_cross_entropy(x, w, labels),
    }


@pytest.mark.parametrize("name", ["norm", "route", "rows", "combine", "loss"])
def test_forward_mode_is_refused(tt, name):
    f, x = calls(tt)[name], torch.randn(3, 6)
    with fw.dual_level():
        dual = fw.make_dual(x, torch.ones_like(x))
        with pytest.raises((RuntimeError, NotImplementedError)):
            f(dual)
        with torch.no_grad(), pytest.raises((RuntimeError, NotImplementedError)):
            f(dual)
        f(x)  # no tangents: as ever


@pytest.mark.parametrize("name", ["norm", "route", "rows", "combine", "loss"])
def test_strided_inputs_expanded_gradients_and_second_derivatives(tt, name):
    f = calls(tt)[name]
    wide = torch.randn(6, 3).t().requires_grad_()  # columns apart
    packed = wide.detach().contiguous().requires_grad_()
    a, b = f(wide), f(packed)
    assert torch.equal(a, b)
    (ga,), (gb,) = torch.autograd.grad(a.sum(), wide), torch.autograd.grad(b.sum(), packed)
    assert torch.equal(ga, gb)
    (g,) = torch.autograd.grad((f(packed) ** 2).sum(), packed, create_graph=True)
    with pytest.raises(RuntimeError):  # a second derivative is refused, not left out
        g.sum().backward()


@pytest.mark.parametrize("name", ["norm", "route", "rows", "combine", "loss"])
def test_outputs_can_be_changed_in_place(tt, name):
    f, x = calls(tt)[name], torch.randn(3, 6)
    want, leaf = 2 * f(x), x.clone().requires_grad_()
    got = f(x).mul_(2)
    assert torch.equal(got, want)
    got = f(leaf).mul_(2)
    assert torch.equal(got, want)
    (a,), (b,) = torch.autograd.grad(got.sum(), leaf), torch.autograd.grad(f(leaf).sum() * 2, leaf)
    assert torch.allclose(a, b)


def test_route_gives_its_bias_no_gradient(tt):
    z, bias = torch.randn(5, 6, requires_grad=True), torch.zeros(6, requires_grad=True)
    r = tt.tt_route(z, 2, bias=bias)
    r.weights.sum().backward()
    assert z.grad is not None and bias.grad is None
    assert not any(t.requires_grad for t in r[1:])


def test_experts_layer_on_masked_rows(tt):
    m = tt.TTExperts(8, 12, 6, 2, balance=True, device="cpu")
    x = torch.randn(7, 8, requires_grad=True)
    mask = torch.tensor([True, False] * 3 + [True])
    y = m(x, mask)
    assert torch.equal(y[~mask], x[~mask].detach())  # the residual alone
    y.sum().backward()
    assert all(p.grad is not None for p in m.parameters()) and "balance" in m.state_dict()
    assert torch.allclose(x.grad[~mask], torch.ones(3, 8))
    for bad in (dict(dtype=torch.float64), dict(activation="tanh")):
        with pytest.raises(ValueError):
            tt.TTExperts(8, 12, 6, 2, device="cpu", **bad)


def test_experts_layer_whatever_masked_rows_hold(tt):
    m = tt.TTExperts(8, 12, 6, 2, device="cpu", residual=False)
    x, mask = torch.randn(7, 8), torch.tensor([True, False] * 3 + [True])
    grads = []
    for fill in (0.0, math.nan, math.inf):
        x[~mask] = fill
        leaf = x.clone().requires_grad_()
        y = m(leaf, mask)
        assert not y[~mask].any()
        grads.append(torch.autograd.grad(y[mask].square().sum(), [leaf, *m.parameters()]))
        assert all(torch.equal(a, b) for a, b in zip(grads[0], grads[-1]))
    assert not grads[0][0][~mask].any() and all(bool(g.isfinite().all()) for g in grads[0])


def test_softmax_loss_module(tt):
    head = tt.TTSoftmaxLoss(6, 9, bias=True, ignore_index=2, reduction="sum", device="cpu")
    x = torch.randn(4, 6, requires_grad=True)
    labels = torch.tensor([0, 2, 8, 2])
    loss = head(x, labels)
    z = x.detach() @ head.weight.detach().t()
    want = sum(float(torch.logsumexp(z[i], 0) - z[i, labels[i]]) for i in (0, 2))
    assert math.isclose(float(loss), want, rel_tol=1e-5)
    loss.backward()
    assert not x.grad[[1, 3]].any() and head.weight.grad is not None and head.bias.grad is not None
    with pytest.raises(ValueError):
        tt.TTSoftmaxLoss(6, 9, reduction="max", device="cpu")
