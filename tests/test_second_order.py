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


@pytest.mark.parametrize("wants", ["q", "k", "v", "theta"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention(dtype, wants, monkeypatch):
    # a stand-in that is linear in q, k, v and theta
    monkeypatch.setattr(B, "fwd", lambda q, k, v, alpha, *a, **kw: ((q + 2 * k + 3 * v).detach() * alpha, q.detach()[..., 0].float()))
    monkeypatch.setattr(B, "bwd", lambda q, k, v, lse, do, alpha, *a, **kw: tuple(
        (c * alpha * do).detach() for c in (1, 2, 3)) + (torch.full((1,), 5.0), None))
    monkeypatch.setattr(B, "residuals_like", lambda q, *a: torch.zeros(4, dtype=torch.uint8))
    monkeypatch.setattr(fa.autograd, "alpha_of_theta", lambda theta: 1.0)
    leaves = {n: torch.ones(1, 1, 3, 64, dtype=dtype) for n in "qkv"} | {"theta": torch.tensor(0.25)}
    leaf = leaves[wants].requires_grad_()

    def run():
        return fa.fib_attention(leaves["q"], leaves["k"], leaves["v"], leaves["theta"], [1.0, 2.0], 8).float().sum()

    want = {"q": 1.0, "k": 2.0, "v": 3.0, "theta": 5.0}[wants]
    first, = torch.autograd.grad(run(), leaf)
    assert (first == want).all() and not first.requires_grad
    out = run()
    graph, = torch.autograd.grad(out, leaf, create_graph=True)
    assert torch.equal(graph, first)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (out + graph.float().square().sum()).backward()


def test_theta_may_change_between_forward_and_backward(monkeypatch):
    test_attention(torch.float32, "theta", monkeypatch)
    q, theta = torch.ones(1, 1, 3, 64, requires_grad=True), torch.tensor(0.25, requires_grad=True)
    out = fa.fib_attention(q, q, q, theta, [1.0, 2.0], 8)
    with torch.no_grad():
        theta.add_(1.0)
    out.sum().backward()
    assert theta.grad == 5.0
