"""The dense layers' module side on the CPU: what reaches the library, what is refused, what an optimizer step computes.  The library's calls are
replaced by their plain forms."""
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
    monkeypatch.setattr(binding, "tt_dense_forward", forward)
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
