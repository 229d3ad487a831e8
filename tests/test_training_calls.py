"""Ordinary ways to call the loss head and the clipping from a training loop."""
from __future__ import annotations

import pytest
import torch

import paper_2606_28560_gb300 as fa


def head(n, d, v, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(n, d, generator=g).to(dtype).cuda(), (torch.randn(v, d, generator=g) * 0.3).to(dtype).cuda()
    return x, w, torch.randint(0, v, (n,), generator=g).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("join", [torch.cat, torch.stack])
def test_losses_that_are_joined(join, dtype):
    """The second loss's incoming gradient is a view that starts 20 bytes into the joined one."""
    (x, w, t), weights = head(10, 64, 50, dtype), torch.arange(1.0, 11.0, device="cuda")
    x1, x2 = (x[i:i + 5].clone().requires_grad_() for i in (0, 5))
    parts = [fa.linear_cross_entropy(x1, w, t[:5], reduction="none"), fa.linear_cross_entropy(x2, w, t[5:].clone(), reduction="none")]
    (join(parts).reshape(-1) * weights).sum().backward()
    for part, leaf, at in ((parts[0], x1, 0), (parts[1], x2, 5)):
        alone = x[at:at + 5].clone().requires_grad_()
        (fa.linear_cross_entropy(alone, w, t[at:at + 5].clone(), reduction="none") * weights[at:at + 5].clone()).sum().backward()
        assert torch.equal(leaf.grad, alone.grad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("view", ["rows of odd width", "flat buffer", "columns", "transposed", "strided targets", "shifted"])
def test_views(view, dtype):
    """Views that are no contiguous memory from a 16-byte boundary give what copies of them give, gradients included."""
    n, d, v = 12, 33, 50
    x, w, t = head(n, d, v, dtype)
    if view == "rows of odd width":
        whole_x, whole_w, cut = head(n + 1, d, v, dtype)[0], w, lambda x, w: (x[1:], w)
    elif view == "flat buffer":
        whole_x, whole_w, cut = x, torch.cat([w.new_zeros(1), w.reshape(-1)]), lambda x, w: (x, w[1:].view(v, d))
    elif view == "columns":
        whole_x, whole_w, cut = head(n, 2 * d, v, dtype)[0], head(n, 2 * d, v, dtype)[1], lambda x, w: (x[:, :d], w[:, d:])
    elif view == "transposed":
        whole_x, whole_w, cut = x.t().contiguous(), w.t().contiguous(), lambda x, w: (x.t(), w.t())
    elif view == "strided targets":
        t = torch.stack([t, t], 1)[:, 0]
        whole_x, whole_w, cut = x, w, lambda x, w: (x, w)
    else:                                         # one sequence, predicted from its own positions
        whole_x, whole_w, cut = head(n + 1, d, v, dtype)[0][None], w, lambda x, w: (x[:, 1:], w)
        t = t[None]
    whole_x, whole_w = whole_x.clone().requires_grad_(), whole_w.clone().requires_grad_()
    loss = fa.linear_cross_entropy(*cut(whole_x, whole_w), t)
    loss.backward()
    x, w = (i.detach().contiguous().clone().requires_grad_() for i in cut(whole_x, whole_w))
    want = fa.linear_cross_entropy(x, w, t.contiguous())
    want.backward()
    assert torch.equal(loss, want)
    got = cut(whole_x.grad, whole_w.grad)
    assert torch.equal(got[0], x.grad) and torch.equal(got[1], w.grad)
