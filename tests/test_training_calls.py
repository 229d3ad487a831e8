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


# The norm's relative error: squares in fp32 runs of at most 258 roundings, half of that in the root, and
# its own rounding; an output has the coefficient's and its own (bf16: 2^-9) on top.
NORM_TOL = 131 * 2.0 ** -24


def parameters_with(grads):
    out = []
    for g in grads:
        p = torch.nn.Parameter(torch.zeros_like(g))
        p.grad = g
        out.append(p)
    return out


def check_clipped(grads, max_norm):
    """Clips, and compares with the definition in 64 bits."""
    keep = [g.detach().clone().double().cpu() for g in grads]
    total = sum(float(k.square().sum()) for k in keep) ** 0.5
    coef = min(1.0, max_norm / (total + 1e-6))
    params = parameters_with(grads)
    norm = fa.clip_grad_norm_(iter(params), max_norm)
    assert norm.dtype == torch.float32 and norm.shape == () and abs(float(norm) - total) <= NORM_TOL * total
    for p, g, k in zip(params, grads, keep):
        assert p.grad is g
        tol = 2.0 ** -8 if g.dtype == torch.bfloat16 else NORM_TOL + 2.0 ** -22
        assert ((g.double().cpu() - k * coef).abs() <= tol * (k * coef).abs() + 1e-37).all()
    return norm


@pytest.mark.gpu
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clipping_with_gradients_on_the_cpu(max_norm):
    """A model's layers on the GPU and its thetas on the CPU."""
    g = torch.Generator().manual_seed(4)
    grads = [torch.randn(33, 65, generator=g).cuda(), torch.randn((), generator=g), torch.randn(1000, generator=g).bfloat16().cuda(),
             torch.randn((), generator=g), torch.randn(7, generator=g)]
    assert check_clipped(grads, max_norm).is_cuda


@pytest.mark.gpu
def test_clipping_a_model_with_its_thetas_on_the_cpu():
    layers = [fa.FibAttention(W=8, theta=0.1 * i) for i in range(2)]
    up = torch.nn.Linear(64, 64, device="cuda")
    q = torch.randn(1, 2, 50, 64, generator=torch.Generator().manual_seed(5)).cuda()
    x = up(q)
    for a in layers:
        x = a(x, x, x)
    x.square().sum().backward()
    params = [*up.parameters(), *(a.theta for a in layers)]
    assert not layers[0].theta.is_cuda and layers[0].theta.grad is not None
    check_clipped([p.grad for p in params], 0.25)


def test_clipping_on_the_cpu_alone_is_refused():
    with pytest.raises(ValueError, match="CUDA"):
        fa.clip_grad_norm_(parameters_with([torch.ones(3)]), 1.0)


LAYOUTS = {
    "transposed": lambda t: t(40, 70).t(),
    "channels last": lambda t: t(2, 5, 6, 3).permute(0, 3, 1, 2),
    "permuted": lambda t: t(3, 1, 4, 9).permute(2, 0, 3, 1),
    "columns": lambda t: t(40, 70)[:, 3:20],
    "every other": lambda t: t(501)[::2],
    "none": lambda t: t(0, 7).t(),
    "on the CPU, transposed": lambda t: t(4, 7).cpu().t(),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_clipping_gradients_of_any_layout(layout, max_norm, dtype):
    g = torch.Generator().manual_seed(6)
    whole = []

    def make(*shape):
        whole.append(torch.randn(*shape, generator=g).to(dtype).cuda())
        return whole[-1]

    grads = [make(100), LAYOUTS[layout](make), make(3, 5)]
    base = grads[1]._base if grads[1]._base is not None else grads[1]
    outside = torch.ones_like(base, dtype=torch.bool)
    torch.as_strided(outside, grads[1].shape, grads[1].stride(), grads[1].storage_offset()).fill_(False)
    keep = base.clone()
    check_clipped(grads, max_norm)
    assert torch.equal(base[outside], keep[outside])


@pytest.mark.gpu
def test_clipping_gradients_in_the_order_of_their_memory_makes_no_copies(monkeypatch):
    """A permutation of contiguous memory is clipped where it lies."""
    seen = []
    real = fa.training.B.clip_grads
    monkeypatch.setattr(fa.training.B, "clip_grads", lambda g, m: seen.append([t.data_ptr() for t in g]) or real(g, m))
    grads = [torch.randn(40, 70, device="cuda").t(), torch.randn(2, 5, 6, 3, device="cuda").permute(0, 3, 1, 2)]
    check_clipped(grads, 0.5)
    assert seen[-1] == [t.data_ptr() for t in grads]


def test_the_norm_of_no_gradients_is_where_the_parameters_are():
    def device_of(*parameters):
        norm = fa.clip_grad_norm_(iter(parameters), 1.0)
        assert norm.shape == () and norm.dtype == torch.float32
        return norm.device.type

    cpu, meta = torch.nn.Parameter(torch.zeros(3)), torch.nn.Parameter(torch.zeros(3, device="meta"))   # meta: any device but the CPU
    assert device_of() == "cpu" and device_of(cpu) == "cpu" and device_of(cpu, meta) == "meta"
    assert float(fa.clip_grad_norm_(cpu, 1.0)) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("fp32", ["x", "w"])
def test_types_that_differ_under_autocast(fp32):
    x, w, t = head(20, 64, 50, torch.bfloat16)
    x, w = (v.float().requires_grad_() if n == fp32 else v.requires_grad_() for n, v in (("x", x), ("w", w)))
    with torch.autocast("cuda", dtype=torch.bfloat16):
        loss = fa.linear_cross_entropy(x, w, t)
    loss.backward()
    x2, w2 = (v.detach().bfloat16().requires_grad_() for v in (x, w))
    want = fa.linear_cross_entropy(x2, w2, t)
    want.backward()
    assert torch.equal(loss, want) and x.grad.dtype == x.dtype and w.grad.dtype == w.dtype
    assert torch.equal(x.grad.float(), x2.grad.float()) and torch.equal(w.grad.float(), w2.grad.float())
    for context in (torch.autocast("cuda", dtype=torch.float16), torch.autocast("cuda", enabled=False)):
        with context, pytest.raises(ValueError, match="one dtype"):
            fa.linear_cross_entropy(x, w, t)


@pytest.mark.gpu
def test_fp32_stays_fp32_under_autocast():
    x, w, t = head(20, 64, 50, torch.float32)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        loss = fa.linear_cross_entropy(x, w, t)
    assert torch.equal(loss, fa.linear_cross_entropy(x, w, t))
