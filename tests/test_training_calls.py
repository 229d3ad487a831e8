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
