"""The example model generating: its layers over the library's paged cache."""
from __future__ import annotations

import warnings

import pytest
import torch

import paper_2606_28560_gb300 as fa
from tests.test_training_example import load


@pytest.mark.gpu
def test_steps_are_the_model():
    """Prompts in two pieces and single tokens, in fp32: the states of the whole
    sequence.  A layer's attention is within 1e-4 of the definition both ways; norms and
    products of 128 random weights of one layer keep that below 1e-3 of the state."""
    m = load()
    torch.manual_seed(1)
    model = m.Model(2, 128).cuda()
    tokens = torch.randint(0, 256, (3, 50)).cuda()
    with torch.no_grad():
        want = model.states(tokens)
        caches, at, got = model.caches(50, 3, torch.float32), 0, []
        for n in (20, 1, 1, 27, 1):
            positions = torch.arange(at, at + n, device="cuda", dtype=torch.int32).repeat(3)
            seqs = torch.arange(3, device="cuda", dtype=torch.int32).repeat_interleave(n)
            got.append(model.steps(tokens[:, at:at + n].reshape(-1), caches, positions, seqs, model.alphas()).view(3, n, -1))
            at += n
    got = torch.cat(got, 1)
    assert float((got - want).norm() / want.norm()) <= 1e-3
    assert fa.check_status() == 0


@pytest.mark.gpu
def test_generates():
    m = load()
    torch.manual_seed(1)
    model = m.Model(2, 128).cuda()
    prompts = torch.randint(0, 256, (2, 33)).cuda()
    text = model.generate(prompts, 40)
    assert text.shape == (2, 40) and int(text.min()) >= 0 and int(text.max()) < 256
    assert torch.equal(model.generate(prompts[1:], 7)[0], model.generate(prompts[1:], 40)[0, :7])
    assert fa.check_status() == 0


def test_generates_nothing():
    model = load().Model(1, 64)
    text = model.generate(torch.zeros(2, 5, dtype=torch.int64), 0)
    assert text.shape == (2, 0) and text.dtype == torch.int64


@pytest.mark.gpu
def test_generated_bytes_are_the_likeliest():
    """Each byte that `generate` chose has, by the states of the whole text, the largest logit
    that there is, as far as both paths may differ: six roundings of at most 2^-8 (of bf16 values
    that fall to different sides) in each of two layers, whose random products enlarge an error no
    more than what they are given: 12 2^-8 of the state's norm and as much of a logit's bound
    |x| |e|, for the byte and for the largest.  Over 1 % of the bytes pass that bound where a state is
    taken one byte early or a position is off by one: 480 of them."""
    m = load()
    torch.manual_seed(3)
    model = m.Model(2, 128).cuda()
    prompts, n = torch.randint(0, 256, (8, 33)).cuda(), 60
    text = model.generate(prompts, n)
    with torch.no_grad():
        with torch.autocast("cuda", dtype=torch.bfloat16):
            x = model.states(torch.cat([prompts, text], 1))[:, 32:-1]
        logits = x.float() @ model.embedding.float().t()
        margin = 2 * 12 * 2.0 ** -8 * x.float().norm(dim=-1) * model.embedding.norm(dim=-1).max()
    chosen = logits.gather(2, text[..., None])[..., 0]
    assert text.shape == (8, n) and (chosen >= logits.amax(-1) - margin).all()
    assert fa.check_status() == 0


@pytest.mark.gpu
def test_layer_over_a_cache():
    """The module's call, for tokens and for a tree, is the library's; another rotation is refused."""
    layer = fa.FibAttention(W=5, theta=0.3, scale=0.2, dedup=False).cuda()
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    cache = fa.PagedCache.empty(4, 8, 2, table, dtype=torch.float32)
    positions = torch.arange(30, dtype=torch.int32, device="cuda")
    seqs = torch.zeros(30, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(30, h, 64, device="cuda") for h in (4, 2, 2))
    fa.cache_append(cache, k, v, positions, seqs=seqs)
    q.requires_grad_()
    out, lse = layer.cached(q, cache, positions, seqs=seqs)
    whole = layer(*(t.detach().transpose(0, 1)[None].contiguous() for t in (q, k, v)))
    assert not out.requires_grad and (out - whole[0].transpose(0, 1)).abs().max() <= 2e-4
    parents = positions - 1
    tree = layer.cached(q, cache, positions, seqs=seqs, parents=parents, slots=positions, alpha=layer.alpha)
    assert torch.equal(tree[0], out) and torch.equal(tree[1], lse)
    with pytest.raises(ValueError, match="parents and slots"):
        layer.cached(q, cache, positions, seqs=seqs, parents=parents)
    with pytest.raises(ValueError, match="rope_base"):
        layer.cached(q, fa.PagedCache.empty(4, 8, 2, table, dtype=torch.float32, rope_base=5e5), positions, seqs=seqs)


@pytest.mark.gpu
def test_layer_in_a_capture():
    """With alpha given, the layer's call is captured; without, theta would be read from the
    GPU: refused, and the capture goes on."""
    layer = fa.FibAttention(W=5, theta=0.3).cuda()
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    cache = fa.PagedCache.empty(4, 8, 2, table, dtype=torch.float32)
    positions = torch.arange(30, dtype=torch.int32, device="cuda")
    seqs = torch.zeros(30, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(30, h, 64, device="cuda") for h in (4, 2, 2))
    fa.cache_append(cache, k, v, positions, seqs=seqs)
    alpha = layer.alpha
    want = layer.cached(q, cache, positions, seqs=seqs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="alpha"):
            layer.cached(q, cache, positions, seqs=seqs)
        got = layer.cached(q, cache, positions, seqs=seqs, alpha=alpha)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    fixed = fa.FibAttention(W=5, theta=0.3, learned=False)           # theta on the CPU: read without waiting
    torch.cuda.synchronize()
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        got = fixed.cached(q, cache, positions, seqs=seqs)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_alpha_is_read_without_a_warning():
    layer, always = fa.FibAttention(theta=0.3), torch.is_warn_always_enabled()
    torch.set_warn_always(True)
    try:
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            assert abs(layer.alpha - 1.0744425) < 1e-6
    finally:
        torch.set_warn_always(always)
