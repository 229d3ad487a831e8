"""The operators that follow a language model's last layer in a training step,
as workloads: the cross-entropy loss of a linear head over a large vocabulary
(``linear_xent_fwd`` / ``linear_xent_bwd``) and the global gradient norm with
clipping (``clip_grads``).

Every case can be run in two forms on the same inputs: the plain form, in
elementary torch operations in 32 bits, and (with ``own`` set) the calls of
this library.  ``exact`` gives the same outputs in 64 bits.

A cross-entropy case: x [N, D] hidden states, w [V, D] head weights (the tied
embedding), one target per row, -100 marking a row without one.  "score"
returns the loss and the log of the softmax normaliser per row; "step" also
returns the gradients of sum_n dloss[n] * loss[n] by x and w.

A clipping case: gradients of the parameters of a model of ``layers`` layers
and width ``hidden`` over ``vocab`` tokens (the paper's host architecture:
grouped-query attention, gated feed-forward, tied embedding, one scalar per
layer), views of one flat buffer per type, clipped into views of another.
"""
import math

import torch

own = False

IGNORE = -100
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases ----

def _xent(name, what, dtype, n, d, v, masked=0.0):
    return {"name": name, "op": "xent", "what": what, "dtype": dtype, "n": n, "d": d, "v": v, "masked": masked}


def _clip(name, dtype, layers, hidden, vocab, norm):
    return {"name": name, "op": "clip", "dtype": dtype, "layers": layers, "hidden": hidden, "vocab": vocab,
            "norm": norm}


def listed():
    return [
        # log-probability of the one token that a decoding step has chosen
        _xent("score one token", "score", "bf16", 1, 512, 32768),
        # perplexity of one sequence of the length-extrapolation workload
        _xent("score a sequence", "score", "bf16", 4096, 512, 32768),
        # odd sizes in fp32, as in a small study; a quarter of the rows is padding
        _xent("score odd sizes f32", "score", "f32", 1001, 100, 5003, 0.25),
        # a byte-level toy model's step
        _xent("step of a toy model", "step", "bf16", 100, 64, 257),
        # the training step's loss: 16 sequences of 1024 tokens, hidden 512, vocabulary 32768
        _xent("step of 16 sequences", "step", "bf16", 16384, 512, 32768),
        # fp32 training of two sequences
        _xent("step in f32", "step", "f32", 2048, 512, 32768),
        # fine-tuning: the prompt's half of the rows carries no target, no size is round
        _xent("step of ragged sizes", "step", "bf16", 3001, 712, 20011, 0.5),
        # a wider model with twice the vocabulary
        _xent("step of a wide model", "step", "bf16", 16384, 1024, 65536),
        # a toy model's gradients (some 200 thousand values, norm below the limit: copied)
        _clip("clip a toy model", "f32", 2, 64, 257, 0.5),
        # the 60M model's gradients in fp32, clipped to 1
        _clip("clip 60M in f32", "f32", 16, 512, 32768, 3.0),
        # odd widths: no tensor but the first starts on a 16-byte boundary
        _clip("clip odd widths", "bf16", 12, 333, 10007, 3.0),
        # a model of about a billion parameters in bf16
        _clip("clip 1B in bf16", "bf16", 20, 2048, 65536, 3.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        dtype = rng.choice(["bf16", "f32"])
        while True:
            c = _clip("", dtype, rng.randint(1, 24), _log_uniform(rng, 32, 2048), _log_uniform(rng, 100, 65536),
                      rng.choice([0.5, 3.0]))
            if sum(_numels(c)) * TYPES[dtype].itemsize <= 2_000_000_000:
                break
    else:
        what, dtype = rng.choice(["score", "step"]), rng.choice(["bf16", "bf16", "f32"])
        while True:
            n, d, v = _log_uniform(rng, 1, 32768), _log_uniform(rng, 64, 2048), _log_uniform(rng, 100, 131072)
            if rng.random() < 0.5:
                d = max(64, d // 64 * 64)
            if n * d * v <= (2 ** 39 if dtype == "bf16" else 2 ** 36):
                break
        c = _xent("", what, dtype, n, d, v, rng.choice([0.0, 0.0, 0.25, 0.9, 1.0]))
    del c["name"]
    return c


def _numels(c):
    """Parameter sizes in the order of a module's parameters()."""
    h, f = c["hidden"], c["hidden"] * 8 // 3
    kv = max(1, h // 4)
    layer = [1, h, h * h, h * kv, h * kv, h * h, h, h * f, h * f, f * h]   # theta, norm, q, k, v, o, norm, gate, up, down
    return [c["vocab"] * h] + layer * c["layers"] + [h]


# ----------------------------------------------------------------- inputs ----

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    if case["op"] == "xent":
        n, d, v = case["n"], case["d"], case["v"]
        # token frequencies fall with the rank; hidden states lean towards their target's row, as a trained model's do
        targets = torch.rand(n, generator=g, device="cuda").mul_(math.log(v)).exp_().long().clamp_(1, v).sub_(1)
        w = torch.randn(v, d, generator=g, device="cuda").mul_(2.0 / math.sqrt(d))
        lean = torch.rand(n, 1, generator=g, device="cuda").mul_(2.0)
        x = torch.randn(n, d, generator=g, device="cuda") + lean * w[targets]
        drop = torch.rand(n, generator=g, device="cuda") < case["masked"]
        targets = torch.where(drop, torch.full_like(targets, IGNORE), targets)
        kept = (targets != IGNORE).sum().clamp(min=1)
        dloss = torch.where(drop, 0.0, 1.0 / kept).float()
        return {"case": case, "x": x.to(dtype), "w": w.to(dtype), "targets": targets, "dloss": dloss}
    sizes = _numels(case)
    total = sum(sizes)
    flat = torch.empty(total, dtype=dtype, device="cuda")
    step = 1 << 26
    for at in range(0, total, step):
        m = min(step, total - at)
        flat[at:at + m] = torch.randn(m, generator=g, device="cuda").mul_(case["norm"] / math.sqrt(total))
    out = torch.empty_like(flat)
    return {"case": case, "grads": list(flat.split(sizes)), "outs": list(out.split(sizes)), "out": out, "max_norm": 1.0}


# ------------------------------------------------------------- plain forms ----

def _plain_xent(x, w, targets, dloss, step):
    xf, wf = x.float(), w.float()
    rows = torch.arange(x.shape[0], device=x.device)
    valid = targets != IGNORE
    at = torch.where(valid, targets, 0)
    s = xf @ wf.t()
    m = s.amax(1, keepdim=True)
    e = torch.exp(s - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total)).squeeze(1)
    loss = torch.where(valid, lse - s[rows, at], 0.0)
    if not step:
        return {"loss": loss, "lse": lse}
    g = torch.where(valid, dloss, 0.0)
    ds = e.mul_((g / total.squeeze(1)).unsqueeze(1))
    ds[rows, at] -= g
    return {"loss": loss, "lse": lse, "dx": (ds @ wf).to(x.dtype), "dw": (ds.t() @ xf).to(w.dtype)}


def _plain_clip(grads, out, max_norm):
    flat = torch.cat([t.reshape(-1) for t in grads]).float()
    norm = flat.square().sum().sqrt()
    coef = (max_norm / (norm + 1e-6)).clamp(max=1.0)
    out.copy_(flat * coef)
    return {"norm": norm, "out": out}


def run(state):
    c = state["case"]
    if c["op"] == "xent":
        x, w, t, step = state["x"], state["w"], state["targets"], c["what"] == "step"
        if not own:
            return _plain_xent(x, w, t, state["dloss"], step)
        import paper_2606_28560_gb300 as fa
        loss, lse = fa.linear_xent_fwd(x, w, t, ignore_index=IGNORE)
        if not step:
            return {"loss": loss, "lse": lse}
        dx, dw = fa.linear_xent_bwd(x, w, t, lse, state["dloss"], ignore_index=IGNORE)
        return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}
    if not own:
        return _plain_clip(state["grads"], state["out"], state["max_norm"])
    import paper_2606_28560_gb300 as fa
    norm = fa.clip_grads(state["grads"], state["max_norm"], out=state["outs"])
    return {"norm": norm, "out": state["out"]}


def work(case):
    es = TYPES[case["dtype"]].itemsize
    if case["op"] == "xent":
        n, d, v = case["n"], case["d"], case["v"]
        once = (n * d + v * d) * es + n * (8 + 4 + 4)       # x, w, targets in; loss, lse out
        if case["what"] == "score":
            return {"bytes": once, "flops": 2 * n * d * v}
        return {"bytes": once + n * 4 + (n * d + v * d) * es, "flops": 6 * n * d * v}
    total = sum(_numels(case))
    return {"bytes": 2 * total * es + 4, "flops": 3 * total}


# ------------------------------------------------------------------- exact ----

def exact(case, seed):
    """The definitions in 64 bits, a block of rows (of values) at a time."""
    s = prepare(case, seed)
    if case["op"] == "clip":
        sq = sum(float(t.double().pow(2).sum()) for t in s["grads"])
        norm = math.sqrt(sq)
        coef = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor(norm, dtype=torch.float64),
                "out": torch.cat([t.reshape(-1).double() * coef for t in s["grads"]])}
    w, step = s["w"].double(), case["what"] == "step"
    loss, lse, dx = [], [], []
    dw = torch.zeros_like(w) if step else None
    block = max(1, min(case["n"], 2 ** 28 // case["v"]))
    for a in range(0, case["n"], block):
        x, t, g = (s[k][a:a + block] for k in ("x", "targets", "dloss"))
        x, g = x.double(), g.double()
        logits = torch.einsum("nd,vd->nv", x, w)
        z = torch.logsumexp(logits, dim=1)
        has = t.ne(IGNORE)
        one = torch.zeros_like(logits)
        one[has.nonzero().squeeze(1), t[has]] = 1.0
        lse.append(z)
        loss.append((z - (logits * one).sum(1)) * has)
        if step:
            ds = (torch.exp(logits - z[:, None]) - one) * (g * has)[:, None]
            dx.append(torch.einsum("nv,vd->nd", ds, w))
            dw += torch.einsum("nv,nd->vd", ds, x)
    got = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    if step:
        got |= {"dx": torch.cat(dx), "dw": dw}
    return got
