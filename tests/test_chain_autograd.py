"""How the differentiable operators meet autograd (CPU): what stands for the kernels here
is torch's own."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2002_06115_amd import chain


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(chain, "_embed_forward", lambda table, ids, offsets, scale, pool:
                        (table.detach()[ids] * scale, table.shape[0], None, 0))
    monkeypatch.setattr(chain, "_constrain_forward", lambda z, bias, *rest:
                        (z.detach() + (0 if bias is None else bias.detach()[:, None]), 0,
                         chain._Limits(repeat_all=1.0)))


def test_forward_mode_is_refused(plain):
    """A tensor with a tangent: without the refusal its derivative would be lost."""
    table, ids = torch.randn(5, 3), torch.tensor([0, 4])
    z, bias = torch.randn(5, 3), torch.randn(5)
    for mode in (torch.enable_grad, torch.no_grad):
        with mode(), forward_ad.dual_level():
            dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
            for call in (lambda: chain.embed(dual(table), ids),
                         lambda: chain.constrain(dual(z)),
                         lambda: chain.constrain(dual(z), bias=bias),
                         lambda: chain.constrain(z, bias=dual(bias))):
                with pytest.raises((RuntimeError, NotImplementedError)):
                    call()
            assert torch.equal(chain.embed(table, ids), table[ids])
            assert torch.equal(chain.constrain(z, bias=bias), z + bias[:, None])


def test_no_graph_without_a_gradient(plain):
    table, ids = torch.randn(5, 3).requires_grad_(), torch.tensor([0, 4])
    z, bias = torch.randn(5, 3), torch.randn(5).requires_grad_()
    assert chain.embed(table, ids).requires_grad
    assert chain.constrain(z, bias=bias).requires_grad
    assert not chain.embed(table.detach(), ids).requires_grad
    assert not chain.constrain(z, bias=bias.detach()).requires_grad
    with torch.no_grad():
        assert not chain.embed(table, ids).requires_grad
        assert not chain.constrain(z, bias=bias).requires_grad
    with torch.inference_mode():
        assert not chain.embed(table, ids).requires_grad


class _Hop:
    """A KB's two calls in torch: Y = X * R's sum, elementwise enough for a graph."""
    def follow(self, X, R, residual=None):
        return X.detach() * R.detach().sum(0)

    def follow_backward(self, X, R, dY, want_dx=True, want_dr=True, residual=None):
        return (dY * 2.0 if want_dx else None), (X if want_dr else None)


def test_sets_are_packed_only_for_a_backward_pass(monkeypatch):
    import types
    import paper_2002_06115_amd as kbf
    packed = []

    def pack(X):
        packed.append(X)
        return types.SimpleNamespace(data=X.detach().clone())

    monkeypatch.setattr(kbf, "_packed", pack)
    monkeypatch.setattr(kbf, "Packed", lambda data, b: data)
    X, R = torch.ones(2, 3), torch.ones(2, 3)
    for leaf in (X.clone().requires_grad_(), X):
        R_leaf = R.clone().requires_grad_()
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                for follow in (kbf.follow, kbf.follow_residual):
                    assert torch.equal(follow(_Hop(), leaf, R_leaf, pack=True), 2 * X)
        assert not packed
        Y = kbf.follow(_Hop(), leaf, R_leaf, pack=True)
        assert len(packed) == 1
        Y.sum().backward()
        assert torch.equal(R_leaf.grad, X)
        packed.clear()
    leaf = X.clone().requires_grad_()
    kbf.follow(_Hop(), leaf, R, pack=True).sum().backward()  # dX needs no set
    assert not packed and torch.equal(leaf.grad, 2 * X)
