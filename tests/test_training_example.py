"""The example training program: attention, loss and clipping together."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import paper_2606_28560_gb300 as fa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("train_bytes", os.path.join(ROOT, "examples", "train_bytes.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
def test_training_learns():
    losses, norms, bits = load().train(steps=40, log=None)
    # uniform bytes cost log 256 = 5.55 nats; text that has been seen for a few steps far less
    assert 5.0 < losses[0] < 6.5 and losses[-1] < losses[0] - 2.0 and bits < 6.5
    assert all(n == n and n > 0 for n in norms)


@pytest.mark.gpu
def test_one_step_against_torch():
    """The same model's loss and gradients with torch's own cross entropy and
    clipping.  The two differ by the bf16 roundings of the logits and of g (torch
    forms bf16 logits: 2^-9 of values of some units), hence 2 %."""
    m = load()
    torch.manual_seed(1)
    model = m.Model(1, 128).cuda()
    g = torch.Generator().manual_seed(2)
    tokens, targets = (torch.randint(0, 256, (4, 64), generator=g).cuda() for _ in range(2))
    targets[0, :10] = -100
    loss = model(tokens, targets)
    loss.backward()
    mine = {n: p.grad.clone() for n, p in model.named_parameters() if p.grad is not None}
    model.zero_grad()
    real = fa.linear_cross_entropy
    fa.linear_cross_entropy = lambda x, w, t: torch.nn.functional.cross_entropy(
        (x.float() @ w.float().t()).reshape(-1, w.shape[0]), t.reshape(-1))
    try:
        other = model(tokens, targets)
    finally:
        fa.linear_cross_entropy = real
    other.backward()
    assert abs(float(loss) - float(other)) <= 1e-4
    for n, p in model.named_parameters():
        if p.grad is not None and p.grad.numel() > 1:
            assert float((p.grad - mine[n]).norm()) <= 0.02 * float(p.grad.norm()), n
    keep = [p.grad.clone() for p in model.parameters() if p.grad is not None and p.is_cuda]
    norm = fa.clip_grad_norm_([p for p in model.parameters() if p.is_cuda], 0.1)
    for p, k in zip((p for p in model.parameters() if p.grad is not None and p.is_cuda), keep):
        p.grad.copy_(k)
    want = torch.nn.utils.clip_grad_norm_([p for p in model.parameters() if p.is_cuda], 0.1)
    assert abs(float(norm) - float(want)) <= 1e-5 * float(want)
