"""What follows the layers in a training step: the loss of a linear head over
a large vocabulary, and gradient clipping (arXiv 2606.28560, Section 3, "Model
and training": a tied embedding over 32768 tokens, gradients clipped to 1).
"""
from __future__ import annotations

import torch

from . import binding as B
from .autograd import differentiable_once


class LinearCrossEntropyFunction(torch.autograd.Function):
    """loss[n] = log sum_v exp(x[n] . w[v]) - x[n] . w[targets[n]], 0 where
    targets[n] is ignore_index.  Neither the logits nor their gradient are kept
    between the forward and the backward; gradients flow to x and w, once: a
    second derivative raises."""

    @staticmethod
    def forward(ctx, x, w, targets, ignore_index):
        loss, lse = B.linear_xent_fwd(x, w, targets, ignore_index=ignore_index)
        ctx.save_for_backward(x, w, targets, lse)
        ctx.ignore_index = ignore_index
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, w, targets, lse = ctx.saved_tensors
        want_dx, want_dw = ctx.needs_input_grad[:2]
        dx, dw = B.linear_xent_bwd(x, w, targets, lse, dloss.contiguous(), ignore_index=ctx.ignore_index,
                                   want_dx=want_dx, want_dw=want_dw)
        return *differentiable_once("linear_cross_entropy", (dx, dw), x, w, dloss), None, None


def linear_cross_entropy(x, w, targets, *, ignore_index: int = -100, reduction: str = "mean"):
    """Cross entropy of the logits ``x @ w.T``.  x [..., D] hidden states, w
    [V, D] head weights of the same dtype (fp32 or bf16, CUDA), targets [...]
    int64; views are taken as they are where they are contiguous and start on a
    16-byte boundary, and copied otherwise.  Where x and w differ under bf16
    autocast (hidden states of the layers, an fp32 head), the fp32 one is cast, as
    torch's own linear does.  ``reduction``: "mean" over the rows with a target (NaN
    when there is none, as the mean of nothing is), "sum", or "none" (the shape
    of targets).  The loss is fp32."""
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be 'mean', 'sum' or 'none'")
    if x.shape[:-1] != targets.shape:
        raise ValueError("targets must have x's shape without its last dimension")
    if x.dtype != w.dtype and torch.is_autocast_enabled("cuda") and torch.get_autocast_dtype("cuda") == torch.bfloat16:
        x, w = (t.bfloat16() if t.dtype == torch.float32 else t for t in (x, w))
    flat = targets.reshape(-1).contiguous()
    x, w = (B.aligned(t.contiguous()) for t in (x.reshape(-1, x.shape[-1]), w))
    loss = LinearCrossEntropyFunction.apply(x, w, flat, int(ignore_index))
    if reduction == "none":
        return loss.reshape(targets.shape)
    if reduction == "sum":
        return loss.sum()
    return loss.sum() / (flat != ignore_index).sum()


def clip_grad_norm_(parameters, max_norm: float) -> torch.Tensor:
    """Clips the gradients of ``parameters`` (an iterable, or one tensor) to a
    global norm of ``max_norm`` in place; parameters without a gradient are left
    out.  Returns the norm before clipping, a 0-dim fp32 tensor on the device;
    nothing waits for the GPU, unless gradients are on the CPU (that of a theta
    kept there): those are clipped with the others, through copies, as are those
    whose values do not fill their memory (slices)."""
    if torch.is_tensor(parameters):
        parameters = [parameters]
    parameters = list(parameters)
    grads = [p.grad for p in parameters if p.grad is not None]
    if not grads:                                 # nothing to clip: 0, where the parameters are
        return torch.zeros((), device=next((p.device for p in parameters if p.device.type != "cpu"), "cpu"))
    try:
        return B.clip_grads(grads, max_norm)
    except ValueError:                            # nothing was launched; not all can be passed as they are
        return _clip_elsewhere(grads, max_norm)


def _in_memory_order(g):
    """g with its dimensions in the order of its memory: contiguous if g is any
    permutation of a contiguous tensor (the norm does not care for the order)."""
    return g.permute(sorted(range(g.dim()), key=g.stride, reverse=True))


@torch.no_grad()
def _clip_elsewhere(grads, max_norm):
    device = next((g.device for g in grads if g.is_cuda), "cpu")
    passed, copied = [], []
    for g in grads:
        p = _in_memory_order(g)
        if p.device != device or not p.is_contiguous():
            p = g.to(device).contiguous()
            copied.append((g, p))
        passed.append(p)
    norm = B.clip_grads(passed, max_norm)
    for g, p in copied:
        g.copy_(p)
    return norm
