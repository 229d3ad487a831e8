"""Differentiating a gradient of the library's functions raises instead of
leaving the second order out.  On the CPU: the calls of the library are stand-ins
in torch operations."""
from __future__ import annotations

import pytest
import torch

import paper_2606_28560_gb300 as fa
from paper_2606_28560_gb300 import binding as B


def _fwd(x, w, t, *, ignore_index):
    s = x.detach() @ w.detach().t()
    lse = torch.logsumexp(s, 1)
    return (lse - s.gather(1, t.clamp(min=0)[:, None])[:, 0]) * (t != ignore_index), lse


def _bwd(x, w, t, lse, dloss, *, ignore_index, want_dx, want_dw):
    x, w, dloss = x.detach(), w.detach(), dloss.detach()
    g = torch.exp(x @ w.t() - lse[:, None])
    g[torch.arange(len(t)), t.clamp(min=0)] -= 1.0
    g = g * (dloss * (t != ignore_index))[:, None]
    return g @ w if want_dx else None, g.t() @ x if want_dw else None


@pytest.fixture
def head(monkeypatch):
    monkeypatch.setattr(B, "linear_xent_fwd", _fwd)
    monkeypatch.setattr(B, "linear_xent_bwd", _bwd)
    g = torch.Generator().manual_seed(0)
    x, w = torch.randn(6, 4, generator=g), torch.randn(9, 4, generator=g)
    return x, w, torch.tensor([0, 8, 3, -100, 2, 2])


@pytest.mark.parametrize("wants", ["x", "w", "both"])
@pytest.mark.parametrize("reduction", ["mean", "sum"])
def test_loss_head(reduction, wants, head):
    x, w, t = head
    leaves = [v.requires_grad_() for n, v in (("x", x), ("w", w)) if wants in (n, "both")]
    loss = fa.linear_cross_entropy(x, w, t, reduction=reduction)
    first = torch.autograd.grad(loss, leaves)                      # the first order is as it was
    ref = torch.nn.functional.cross_entropy(x @ w.t(), t, reduction=reduction)
    for a, b in zip(first, torch.autograd.grad(ref, leaves)):
        assert torch.allclose(a, b, atol=1e-6) and not a.requires_grad
    loss = fa.linear_cross_entropy(x, w, t, reduction=reduction)
    graph = torch.autograd.grad(loss, leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(graph, first))
    with pytest.raises(RuntimeError, match="second derivatives"):
        (loss + sum(v.square().sum() for v in graph)).backward()


def test_loss_head_with_a_gradient_that_depends_on_something(head):
    x, w, t = head
    x.requires_grad_()
    scale = torch.ones(6, requires_grad=True)
    loss = fa.linear_cross_entropy(x, w, t, reduction="none")
    dx, = torch.autograd.grad((loss * scale).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        dx.square().sum().backward()
