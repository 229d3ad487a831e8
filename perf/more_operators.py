"""The operators that generate with the attention, as workloads: writing new keys
and values into a paged cache (``cache_append``), the attention of new tokens over
that cache (``cached_fwd``: one token per sequence while generating, chunks of a
prompt before) and the attention of a tree of drafted tokens (``tree_fwd``).

Every case can be run in two forms on the same inputs: the plain form, in
elementary torch operations in 32 bits (angles in 64), and (with ``own`` set) the
calls of this library.  ``exact`` gives the same outputs in 64 bits.

The cache is a pool of pages, [pages, rows of a page, key/value heads, 64], for
rotated keys (fp16 beside bf16 tensors, fp32 beside fp32) and one for values; a
table names the pages of each sequence, in no order.  Tokens of all sequences lie
behind one another in a batch; ``seqs`` and ``positions`` say whose they are and
where.  A query at position p reads the rows at distances 0 .. W and, for every
rung d <= p, the rows at distances floor(d) and floor(d) + 1, interpolated.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

D = 64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
KEYS = {"bf16": torch.float16, "f32": torch.float32}       # rotated keys in the cache


# ------------------------------------------------------------------ cases ----

def _case(name, op, dtype, seqs, new, heads, kv_heads, page, lo, hi, *, ragged=False, W=8, K=15, base="fib", alpha=0.8,
          dedup=True):
    """``seqs`` sequences of lo .. hi tokens in the cache and ``new`` more tokens each (1 .. new if
    ragged); for a tree these are drafts."""
    return {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "new": new, "heads": heads, "kv_heads": kv_heads,
            "page": page, "lo": lo, "hi": hi, "ragged": ragged, "W": W, "K": K, "base": base, "alpha": alpha, "dedup": dedup}


def listed():
    return [
        # one sequence generating: the keys and values of its next token
        _case("append one token", "append", "bf16", 1, 1, 8, 8, 16, 1000, 1000),
        # a server's step: a token for each of 256 sequences, grouped heads (8 over 2)
        _case("append a decoding batch", "append", "bf16", 256, 1, 8, 2, 16, 1, 4000),
        # fp32, three heads, pages of 13 rows, prompts of any length
        _case("append ragged prompts f32", "append", "f32", 7, 800, 3, 3, 13, 0, 50, ragged=True),
        # the prompts of a full batch: 64 sequences of 1024 tokens
        _case("append prompts", "append", "bf16", 64, 1024, 8, 8, 64, 0, 0),
        # one sequence generating: latency
        _case("decode one token", "cached", "bf16", 1, 1, 8, 8, 16, 1500, 1500),
        # 256 sequences of any length, grouped heads
        _case("decode grouped heads", "cached", "bf16", 256, 1, 8, 2, 16, 0, 4000),
        # odd sizes in fp32: window 5, powers of two, every rung kept beside the window
        _case("decode odd sizes f32", "cached", "f32", 33, 1, 6, 3, 13, 0, 700, W=5, K=9, base="pow2", alpha=1.3, dedup=False),
        # a large batch: the cache is read as fast as memory gives it
        _case("decode a large batch", "cached", "bf16", 4096, 1, 8, 8, 64, 64, 2000),
        # chunks of prompts whose beginnings are cached already
        _case("chunks of prompts", "cached", "bf16", 8, 256, 8, 8, 64, 0, 3000),
        # eight drafted tokens of one sequence: latency
        _case("verify eight drafts", "tree", "bf16", 1, 8, 8, 8, 16, 1500, 1500),
        # 64 sequences with 32 drafts each, grouped heads
        _case("verify trees of a batch", "tree", "bf16", 64, 32, 8, 2, 16, 10, 3000),
        # fp32, trees of different sizes, a last page that the tree ends inside
        _case("verify ragged trees f32", "tree", "f32", 19, 50, 3, 3, 13, 0, 500, ragged=True, W=10, alpha=1.4),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max(work(c)["bytes"] for c in listed() if c["op"] == op) for op in ("append", "cached", "tree")}
    op, dtype = rng.choice(["append", "cached", "cached", "tree"]), rng.choice(["bf16", "bf16", "f32"])
    while True:
        kv = rng.choice([1, 2, 3, 4, 8, 8, 16])
        group = rng.choice([1, 1, 2, 3, 4, 8])
        base = rng.choice(["fib", "fib", "pow2"])
        lo = rng.choice([0, 1, _log_uniform(rng, 1, 4000)])
        hi = max(lo, _log_uniform(rng, 1, 8000))
        new = {"append": rng.choice([1, _log_uniform(rng, 1, 1500)]), "cached": rng.choice([1, 1, _log_uniform(rng, 2, 300)]),
               "tree": _log_uniform(rng, 2, 64)}[op]
        c = _case("", op, dtype, _log_uniform(rng, 1, 4096), new, kv * group, kv, _log_uniform(rng, 1, 256), lo, hi,
                  ragged=rng.random() < 0.5, W=rng.randint(0, 16), K=rng.randint(0, 15 if base == "fib" else 10), base=base,
                  alpha=rng.choice([0.5, 1.0, 1.5, round(rng.uniform(0.5, 1.5), 3)]), dedup=rng.random() < 0.7)
        pool = c["seqs"] * (c["hi"] + c["new"] + c["page"]) * kv * D * 2 * TYPES[dtype].itemsize
        if c["seqs"] * c["new"] <= 65536 and pool <= 12_000_000_000 and work(c)["bytes"] <= most[op] and \
                work(c)["flops"] <= max(work(x)["flops"] for x in listed() if x["op"] == op):
            break
    del c["name"]
    return c


@functools.lru_cache(maxsize=64)
def _plan(items):
    """What follows from the case alone: per token its sequence, position, storage slot and parent."""
    c = dict(items)
    rng = random.Random(repr(sorted(items)))
    seqs, positions, slots, parents, ends, deepest = [], [], [], [], [], 0
    for b in range(c["seqs"]):
        have, new = rng.randint(c["lo"], c["hi"]), rng.randint(1, c["new"]) if c["ragged"] else c["new"]
        first, depth = len(seqs), []
        for t in range(new):
            # drafts: mostly children of the last few drafted tokens, some beside the root
            up = -1 if t == 0 or rng.random() < 0.1 else rng.randint(max(0, t - 6), t - 1)
            if c["op"] == "tree":
                depth.append(0 if up < 0 else depth[up] + 1)
                parents.append(up if up < 0 else first + up)
            else:
                depth.append(t)
            seqs.append(b)
            positions.append(have + depth[t])
            slots.append(have + t)
        deepest = max(deepest, max(depth))
        ends.append(have + new)
    return seqs, positions, slots, parents, ends, deepest


def _plan_of(case):
    return _plan(tuple(sorted((k, v) for k, v in case.items() if k != "name")))


def _rungs(case):
    """(floor, weight of the far row) of every rung that is attended beside the window."""
    f = [1, 2]
    while len(f) < case["K"]:
        f.append(f[-1] + f[-2])
    f = f[:case["K"]] if case["base"] == "fib" else [2 ** k for k in range(case["K"])]
    d = np.float32(case["alpha"]) * np.array(f, dtype=np.float32)
    if case["dedup"]:
        d = d[d > case["W"]]
    lo = np.floor(d)
    return lo.astype(np.int64), (d - lo).astype(np.float32)


# ----------------------------------------------------------------- inputs ----

def _normal(g, shape, dtype):
    """Normal values, drawn a part at a time (pools take gigabytes)."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    step = 1 << 28
    for at in range(0, flat.numel(), step):
        m = min(step, flat.numel() - at)
        flat[at:at + m] = torch.randn(m, generator=g, device="cuda")
    return t


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, page, kv, heads = TYPES[case["dtype"]], case["page"], case["kv_heads"], case["heads"]
    seqs, positions, slots, parents, ends, deepest = _plan_of(case)
    n = len(seqs)
    need = [(e + page - 1) // page for e in ends]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((len(ends), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    i32 = {"dtype": torch.int32, "device": "cuda"}
    state = {"case": case, "table": table.cuda(), "k_pages": _normal(g, (pages, page, kv, D), KEYS[case["dtype"]]),
             "v_pages": _normal(g, (pages, page, kv, D), dtype), "seqs": torch.tensor(seqs, **i32),
             "positions": torch.tensor(positions, **i32)}
    # queries, keys and values are views of the layer's one projection
    qkv = _normal(g, (n, (heads + 2 * kv) * D), dtype)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([heads * D, kv * D, kv * D], dim=1))
    state |= {"k": k, "v": v} if case["op"] == "append" else {"q": q}
    lo, far = _rungs(case)
    if case["op"] == "tree":
        state |= {"slots": torch.tensor(slots, **i32), "parents": torch.tensor(parents, **i32), "deepest": deepest}
    # the distances and weights of the attended set, as a program keeps them for its layer
    state["near"] = torch.cat([torch.arange(case["W"] + 1), torch.from_numpy(lo)]).cuda()
    state["weight"] = torch.cat([torch.zeros(case["W"] + 1), torch.from_numpy(far)]).cuda()
    if own:
        import paper_2606_28560_gb300 as fa
        state["cache"] = fa.PagedCache(state["k_pages"], state["v_pages"], state["table"])
        state["offsets"] = fa.base(case["base"], case["K"])
    return state


# ------------------------------------------------------------- plain forms ----

def _rotate(x, positions):
    """x [N, heads, 64] in fp32, pairs (m, m + 32), angle position * 10000^(-m/32)."""
    m = torch.arange(D // 2, device=x.device, dtype=torch.float64)
    angle = positions.double()[:, None] * torch.exp(m * (-math.log(1e4) / (D // 2)))
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _rows(table, seqs, slots, page):
    """Rows of the pool, counted through its pages, of storage slots [N, ...]."""
    shape = [-1] + [1] * (slots.dim() - 1)
    s = slots.long()
    return table[seqs.long().view(shape), s // page].long() * page + s % page


def _plain_append(s):
    page = s["case"]["page"]
    rows = _rows(s["table"], s["seqs"], s["positions"], page)
    k, v = s["k_pages"], s["v_pages"]
    k.view(-1, *k.shape[2:])[rows] = _rotate(s["k"].float(), s["positions"]).to(k.dtype)
    v.view(-1, *v.shape[2:])[rows] = s["v"]
    return {"k_pages": k, "v_pages": v}


def _plain_attention(s):
    c, page = s["case"], s["case"]["page"]
    q, pos, kv = s["q"], s["positions"].long(), c["kv_heads"]
    n, heads = q.shape[:2]
    near, weight = s["near"], s["weight"]
    far = near + (weight > 0)
    valid = far <= pos[:, None]                                       # [N, S]
    if c["op"] == "tree":
        path = [torch.arange(n, device=q.device)]                     # ancestors by distance, -1 beyond the root
        for _ in range(s["deepest"]):
            path.append(torch.where(path[-1] >= 0, s["parents"].long()[path[-1].clamp(min=0)], -1))
        path = torch.stack(path, 1)

    def read(distance):
        at = (pos[:, None] - distance).clamp(min=0)
        if c["op"] == "tree":
            a = path[:, distance.clamp(max=s["deepest"])].masked_fill(distance > s["deepest"], -1)
            at = torch.where(a >= 0, s["slots"].long()[a.clamp(min=0)], at)
        rows = _rows(s["table"], s["seqs"], torch.where(valid, at, torch.zeros_like(at)), page)
        return (p.view(-1, kv, D)[rows].float() for p in (s["k_pages"], s["v_pages"]))

    w = weight[None, :, None, None]
    (k0, v0), (k1, v1) = read(near), read(far)
    k, v = k0 * (1 - w) + k1 * w, v0 * (1 - w) + v1 * w               # [N, S, kv, 64]
    qr = _rotate(q.float(), pos).view(n, kv, heads // kv, D)
    score = (qr @ k.permute(0, 2, 3, 1)) / math.sqrt(D)               # [N, kv, group, S]
    score = score.masked_fill(~valid[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    out = (e @ v.permute(0, 2, 1, 3)) / total
    return {"out": out.reshape(n, heads, D).to(q.dtype), "lse": (top + torch.log(total)).reshape(n, heads)}


def run(state):
    c = state["case"]
    if not own:
        return _plain_append(state) if c["op"] == "append" else _plain_attention(state)
    import paper_2606_28560_gb300 as fa
    cache = state["cache"]
    if c["op"] == "append":
        fa.cache_append(cache, state["k"], state["v"], state["positions"], seqs=state["seqs"])
        return {"k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    if c["op"] == "cached":
        out, lse = fa.cached_fwd(state["q"], cache, c["alpha"], state["offsets"], c["W"], state["positions"],
                                 seqs=state["seqs"], dedup=c["dedup"])
    else:
        out, lse = fa.tree_fwd(state["q"], cache, c["alpha"], state["offsets"], c["W"], state["positions"],
                               state["parents"], state["slots"], seqs=state["seqs"], dedup=c["dedup"])
    return {"out": out, "lse": lse}


def _read_rows(case):
    """(rows of the cache that are read at all, rows read summed over the queries)"""
    seqs, positions, slots, parents, ends, _ = _plan_of(case)
    lo, far = _rungs(case)
    steps = sorted(set(range(case["W"] + 1)) | set(lo.tolist()) | set((lo + 1)[far > 0].tolist()))
    reach = {int(d) + 1 for d, w in zip(lo, far) if w > 0}            # a rung counts from its far row on
    pair = {int(d) for d, w in zip(lo, far) if w > 0}
    whole = set(range(case["W"] + 1)) | {int(d) for d, w in zip(lo, far) if w == 0}
    read, each = set(), 0
    for n, (b, p) in enumerate(zip(seqs, positions)):
        path, at = [], n
        while parents and at >= 0:
            path.append(slots[at])
            at = parents[at]
        for d in steps:
            if (d in whole or d in reach) and d <= p or d in pair and d + 1 <= p:
                read.add((b, path[d] if d < len(path) else p - d))
                each += 1
    return len(read), each


@functools.lru_cache(maxsize=64)
def _work(items):
    case = dict(items)
    n, kv, heads = len(_plan_of(case)[0]), case["kv_heads"], case["heads"]
    es = TYPES[case["dtype"]].itemsize
    if case["op"] == "append":
        return 4 * n * kv * D * es + 12 * n, 3 * n * kv * D            # keys and values in and out, where they go
    rows, each = _read_rows(case)
    ints = (16 if case["op"] == "tree" else 8) * n
    return rows * kv * D * 2 * es + n * heads * (2 * D * es + 4) + ints, 4 * D * each * heads


def work(case):
    size, flops = _work(tuple(sorted((k, v) for k, v in case.items() if k != "name")))
    return {"bytes": size, "flops": flops}


# ------------------------------------------------------------------- exact ----

def _turned(x, positions):
    """The rotation as a product of complex numbers, in 64 bits."""
    theta = 1e4 ** (-torch.arange(0, D, 2, device=x.device, dtype=torch.float64) / D)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), positions.double()[:, None] * theta)
    z = torch.complex(*x.double().chunk(2, dim=-1)) * turn[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    """The definitions in 64 bits, slot by slot."""
    s = prepare(case, seed)
    page, pos, seqs = case["page"], s["positions"].long(), s["seqs"].long()

    def place(slot):                                                  # (page, row within it)
        return s["table"][seqs, slot.div(page, rounding_mode="floor")].long(), slot.remainder(page)

    if case["op"] == "append":
        if s["k_pages"].numel() > 2 ** 31:
            return None
        k, v = s["k_pages"].double(), s["v_pages"].double()
        k[place(pos)], v[place(pos)] = _turned(s["k"], pos), s["v"].double()
        return {"k_pages": k, "v_pages": v}
    lo, far = _rungs(case)
    slots = [(j, 0.0) for j in range(case["W"] + 1)] + [(int(a), float(w)) for a, w in zip(lo, far)]
    n, heads, kv = *s["q"].shape[:2], case["kv_heads"]
    q = _turned(s["q"], pos).view(n, kv, -1, D) * D ** -0.5

    def row(pool, distance, there):
        at = pos - distance
        if case["op"] == "tree":
            a, left = torch.arange(n, device=pos.device), distance
            while left and bool((a >= 0).any()):
                a = torch.where(a < 0, a, s["parents"].long()[a.clamp(min=0)])
                left -= 1
            at = torch.where(a < 0, at, s["slots"].long()[a.clamp(min=0)])
        return pool[place(torch.where(there, at, 0))].double()

    scores, values = [], []
    for near, w in slots:
        there = pos >= (near + 1 if w else near)
        key, value = row(s["k_pages"], near, there), row(s["v_pages"], near, there)
        if w:
            key = key.lerp(row(s["k_pages"], near + 1, there), w)
            value = value.lerp(row(s["v_pages"], near + 1, there), w)
        x = torch.einsum("nkgd,nkd->nkg", q, key)
        scores.append(torch.where(there[:, None, None], x, -math.inf))
        values.append(value)
    lse = torch.logsumexp(torch.stack(scores), 0)
    out = torch.zeros_like(q)
    for x, value in zip(scores, values):
        out += torch.exp(x - lse)[..., None] * value[:, :, None]
    return {"out": out.reshape(n, heads, D), "lse": lse.reshape(n, heads)}
