"""The paged cache: appended keys and values, the attention of new tokens over
them and of trees of drafts, against the definitions in 64 bits, slot by slot.

Tolerances.  u = 2^-24.  A rotated value a c - b s has errors of 2u each in c and
s (the rounded angle and the function) and 3u from its own operations: at most
6u (|a| + |b|), and half a step of its storage type.  A score sums 64 products of
a rotated and scaled query (6u, 3u more) with a stored key in 8 chains of 4 pairs
and a tree of 4: 20u of sum |q d k d| at most, with the slot's interpolation 24u;
A below bounds that sum.  exp2 has 2 ulp and its argument, at most 2A + 1 log2 e
in size, 3 roundings: a weight is off by 2 * 24u A + 6u (A + 1) + 4u of itself,
and so is the sum of weights; values are summed over R rows: (R / 4 + 8) u.
bf16 goes through products of 16-bit halves: those of q keep 22 bits (4u), those of
p 16 (2^-17 = 128u), and a product of 16 may lose of each of its 17 terms what lies
below 2^-24 of the largest: four of them in a score, 4 * 17 u A, and two for 32
rows in a value, (R / 32 + 1) * 34 u V.
"""
from __future__ import annotations

import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2606_28560_gb300 as fa
from paper_2606_28560_gb300 import binding as B
from tests.test_gpu_parity import TOL, bf16_out_tol
from tests.test_binding_devices import library, streams   # noqa: F401 (fixtures)

F32, BF = torch.float32, torch.bfloat16
KEYS = {BF: torch.float16, F32: F32}
U = 2.0 ** -24
D = 64
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------- definitions ----

def rotated(x, positions):
    """R(position) x in 64 bits; x [N, heads, 64]."""
    theta = 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    angle = positions.double()[:, None, None] * theta
    a, b = x.double().chunk(2, dim=-1)
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], dim=-1)


def slots_of(W, alpha, f, dedup=True, round_offsets=False):
    """[(near, weight of the row behind it, distance that has to lie behind the query)]"""
    d = np.float32(alpha) * np.asarray(f, dtype=np.float32)
    if round_offsets:
        d = np.round(d)
    out = [(j, 0.0, j) for j in range(W + 1)]
    for x in d:
        if not dedup or x > W:
            out.append((int(np.floor(x)), float(x - np.floor(x)), float(x)))
    return out


class Model:
    """Caches on the CPU: slots of a sequence by number, [Hkv, 64] each, in 64 bits."""

    def __init__(self, cache):
        self.k, self.v = cache.k_pages.cpu().double(), cache.v_pages.cpu().double()
        self.table, self.rows = cache.block_table.cpu(), cache.k_pages.shape[1]

    def row(self, seq, slot):
        page = int(self.table[seq, slot // self.rows])
        return self.k[page, slot % self.rows], self.v[page, slot % self.rows]

    def attention(self, q, positions, seqs, slots, *, scale=D ** -0.5, parents=None, at=None):
        """out, lse and the bounds A (scores) and V (values) of every token and head."""
        q = rotated(q.cpu(), positions) * scale
        N, H, _ = q.shape
        out, lse = torch.zeros(N, H, D, dtype=torch.float64), torch.full((N, H), -math.inf, dtype=torch.float64)
        A, V = torch.zeros(N, H, dtype=torch.float64), torch.zeros(N, H, dtype=torch.float64)
        for n in range(N):
            p, b = int(positions[n]), int(seqs[n])
            if p < 0 or b < 0:
                continue
            path, cur = [], n
            while parents is not None and cur >= 0:
                path.append(int(at[cur]))
                cur = int(parents[cur])
            keys, values, sizes = [], [], []
            for near, w, need in slots:
                if need > p:
                    continue
                k0, v0 = self.row(b, path[near] if near < len(path) else p - near)
                ka, va = k0.abs(), v0.abs()
                if w:
                    k1, v1 = self.row(b, path[near + 1] if near + 1 < len(path) else p - near - 1)
                    ka, va = (1 - w) * ka + w * k1.abs(), (1 - w) * va + w * v1.abs()
                    k0, v0 = (1 - w) * k0 + w * k1, (1 - w) * v0 + w * v1
                keys.append(k0)
                values.append(v0)
                sizes.append((ka, va))
            G = H // k0.shape[0]                                           # [S, H, 64]
            k, v, ka, va = (torch.stack(t).repeat_interleave(G, 1) for t in (keys, values, *zip(*sizes)))
            s = torch.einsum("hd,shd->sh", q[n], k)
            lse[n] = torch.logsumexp(s, 0)
            out[n] = torch.einsum("sh,shd->hd", torch.exp(s - lse[n]), v)
            A[n] = torch.einsum("hd,shd->sh", q[n].abs(), ka).amax(0)
            V[n] = va.amax((0, 2))
        return out, lse, A, V


def check(got, want, W, K):
    """got: out, lse; want: out, lse, A, V."""
    (out, lse), (ro, rl, A, V) = (t.cpu() for t in got), want
    halves = out.dtype == BF
    score = (24 + halves * (4 + 4 * 17)) * U * A
    weight = 2 * score + 6 * U * (A + 1) + 4 * U
    rows = (W + 1 + 2 * K) / 4 + 8 + halves * (128 + 34 * ((W + 1 + 2 * K) / 32 + 1))
    half = torch.finfo(out.dtype).eps / 2
    err = (out.double() - ro).abs()
    assert (err <= (V * (2 * weight + rows * U))[..., None] * (1 + half) + half * ro.abs()).all(), float(err.max())
    live = rl > -math.inf
    assert torch.equal(lse == -math.inf, ~live)
    err = (lse.double() - rl).abs()[live]
    assert (err <= (weight + 6 * U * (rl.abs() + 1))[live]).all(), float(err.max())


# ------------------------------------------------------------------- setups ----

def tokens(g, N, heads, dtype, extra=0):
    """[N, heads, 64] as a view of a wider projection."""
    return torch.randn(N, (heads + extra) * D, generator=g).to(dtype).cuda().narrow(1, extra * D // 2, heads * D) \
        .unflatten(1, (heads, D))


def pools(layout, pages, rows, Hkv, dtype, fill=float("nan")):
    """Two pools [pages, rows, Hkv, 64], every value `fill`."""
    def one(t):
        if layout == "plain":
            return torch.full((pages, rows, Hkv, D), fill, dtype=t, device="cuda")
        if layout == "heads first":
            return torch.full((pages, Hkv, rows, D), fill, dtype=t, device="cuda").transpose(1, 2)
        if layout == "a layer of several":
            return torch.full((pages, 3, rows, Hkv, D), fill, dtype=t, device="cuda")[:, 1]
        assert layout == "beside others"
        return torch.full((pages, rows, 2, Hkv, D), fill, dtype=t, device="cuda")[:, :, 1]
    return one(KEYS[dtype]), one(dtype)


def filled(lengths, rows, Hkv, dtype, seed, *, layout="plain", more=0):
    """A cache of sequences of `lengths` tokens, with room for `more` each, in pages of
    no order; rows that hold no token are NaN, unused table entries are not pages."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + more + rows - 1) // rows for n in lengths]
    order = torch.randperm(sum(need) + 2, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(need) + 1), -7, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    cache = fa.PagedCache(*pools(layout, sum(need) + 2, rows, Hkv, dtype), table.cuda())
    seqs = torch.cat([torch.full((n,), b) for b, n in enumerate(lengths)]).int()
    positions = torch.cat([torch.arange(n) for n in lengths]).int()
    if len(seqs):
        k, v = (tokens(g, len(seqs), Hkv, dtype, 2) for _ in range(2))
        fa.cache_append(cache, k, v, positions.cuda(), seqs=seqs.cuda())
    return cache, g


def clear():
    try:
        fa.check_status()
    except fa.FibattnError:
        pass


LAYOUTS = ["plain", "heads first", "a layer of several", "beside others"]


# ------------------------------------------------------------------- append ----

@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,Hkv,rows", [(1, 1, 1), (1, 8, 16), (5, 3, 13), (301, 2, 7), (70000, 8, 64), (20000, 19, 5)])
def test_append(N, Hkv, rows, dtype, layout):
    g = torch.Generator().manual_seed(N)
    seqs = (torch.arange(N) * 7 % 3).int()                                  # three sequences, interleaved
    slots = torch.zeros(N, dtype=torch.int32)
    for b in range(3):
        mine = (seqs == b).nonzero()[:, 0]
        slots[mine] = torch.randperm(len(mine), generator=g).int()
    positions = torch.randint(0, 1 << 20, (N,), generator=g).int() if N % 2 else slots.clone()
    M = (N + rows - 1) // rows + 1
    table = torch.randperm(3 * M, generator=g).int().view(3, M)
    pad = torch.zeros(N, dtype=torch.bool)
    pad[3::11] = True
    negative = torch.arange(N) % 2 == 0
    cache = fa.PagedCache(*pools(layout, 3 * M, rows, Hkv, dtype, 0.34375), table.cuda())
    k, v = tokens(g, N, Hkv, dtype, 1), tokens(g, N, Hkv, dtype, 3)
    fa.cache_append(cache, k, v, torch.where(pad & negative, -5, positions).cuda(),
                    seqs=torch.where(pad & ~negative, -1, seqs).cuda(), slots=slots.cuda())
    page = table[seqs.long(), slots.long() // rows].long()
    row = slots.long() % rows
    kp, vp = cache.k_pages.cpu(), cache.v_pages.cpu()
    keep = ~pad
    assert torch.equal(vp[page, row][keep], v.cpu()[keep])
    want = rotated(k.cpu(), positions)[keep]
    a, b = k.cpu().double().abs()[keep].chunk(2, -1)
    tol = (6 * U * (a + b)).repeat(1, 1, 2)
    half = torch.finfo(kp.dtype).eps / 2
    tiny = torch.finfo(kp.dtype).smallest_normal * half
    assert ((kp[page, row][keep].double() - want).abs() <= tol * (1 + half) + half * want.abs() + tiny).all()
    untouched = torch.ones(3 * M, rows, dtype=torch.bool)
    untouched[page[keep], row[keep]] = False
    assert (kp[untouched] == 0.34375).all() and (vp[untouched] == 0.34375).all()
    if layout == "a layer of several":
        assert (cache.k_pages._base[:, ::2] == 0.34375).all() and (cache.v_pages._base[:, ::2] == 0.34375).all()
    if layout == "beside others":
        assert (cache.k_pages._base[:, :, 0] == 0.34375).all() and (cache.v_pages._base[:, :, 0] == 0.34375).all()
    assert fa.check_status() == 0


@pytest.mark.gpu
def test_append_nothing_and_values_as_they_are():
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    cache = fa.PagedCache.empty(1, 4, 2, table)
    cache.k_pages.fill_(1.0)
    fa.cache_append(cache, torch.empty(0, 2, D, dtype=BF, device="cuda"), torch.empty(0, 2, D, dtype=BF, device="cuda"),
                    torch.empty(0, dtype=torch.int32, device="cuda"))
    assert (cache.k_pages == 1.0).all()
    v = torch.arange(2 * D, dtype=torch.int16).view(1, 2, D)                # every kind of bit pattern, NaNs among them
    v = (v * 517 + 0x7f70).to(torch.int16).cuda()
    fa.cache_append(cache, torch.zeros(1, 2, D, dtype=BF, device="cuda"), v.view(BF),
                    torch.tensor([3], dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.v_pages[0, 3].view(torch.int16), v[0])


@pytest.mark.gpu
def test_append_reports_keys_that_fp16_cannot_hold():
    clear()
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    cache = fa.PagedCache.empty(1, 4, 1, table)
    k = torch.zeros(1, 1, D, dtype=BF, device="cuda")
    k[0, 0, 5] = 65000.0
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    fa.cache_append(cache, k, k, at)
    assert fa.check_status() == 0
    k[0, 0, 5] = 70000.0
    fa.cache_append(cache, k, k, at)
    with pytest.raises(fa.FibattnError) as e:
        fa.check_status()
    assert e.value.flags == 2


# ---------------------------------------------------------------- attention ----

FIB, POW = [1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 144, 233, 377, 610, 987], [2.0 ** k for k in range(10)]
SETS = {  # W, alpha, offsets, options
    "usual": (8, 0.8, FIB, {}), "window alone": (4, 1.0, [], {}), "one key": (0, 1.0, [], {}),
    "integers": (8, 1.0, FIB, {}), "every rung": (5, 1.3, POW, {"dedup": False}), "rounded": (2, 0.77, FIB, {"round_offsets": True}),
    "rungs alone": (0, 1.499, [k + 0.4 for k in range(1, 33)], {}), "wide window": (300, 0.9, FIB, {}),
    "the most rows": (1024, 1.0, [1030.5 + 5 * k for k in range(32)], {}),
    "40 rows": (20, 0.8, FIB, {}), "64 rows": (31, 1.1, [32.0 + 3 * k for k in range(16)], {}),
    "65 rows": (32, 1.1, [32.0 + 3 * k for k in range(16)], {}), "dead halves": (0, 1.3, [200.1 + k for k in range(30)], {}),
    "near rungs": (3, 0.6, [0.0, 0.3, 1.0, 1.5, 2.25, 4.0], {"dedup": False}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("which", list(SETS))
@pytest.mark.parametrize("H,Hkv,rows,layout", [(1, 1, 1, "plain"), (8, 8, 16, "plain"), (6, 3, 13, "heads first"),
                                               (8, 1, 64, "a layer of several"), (22, 2, 5, "beside others")])
def test_cached(H, Hkv, rows, layout, which, dtype):
    """Sequences of every length from one token on, one token each and chunks, padding between them."""
    W, alpha, f, opts = SETS[which]
    lengths = [1, 2, 3, 9, 10, 11, 40, 333, 1200]
    cache, g = filled(lengths, rows, Hkv, dtype, H + rows, layout=layout)
    seqs, positions = [], []
    for b, n in enumerate(lengths):
        new = min(n, 1 + b % 4)
        seqs += [b] * new
        positions += range(n - new, n)
    seqs += [-1, 4, 0]
    positions += [3, -1, -2 ** 31]
    order = torch.randperm(len(seqs), generator=g)
    seqs, positions = torch.tensor(seqs).int()[order], torch.tensor(positions).int()[order]
    q = tokens(g, len(seqs), H, dtype, 3)
    got = fa.cached_fwd(q, cache, alpha, f, W, positions.cuda(), seqs=seqs.cuda(), **opts)
    want = Model(cache).attention(q, positions, seqs, slots_of(W, alpha, f, **opts))
    check(got, want, W, len(f))
    assert fa.check_status() == 0
    again = fa.cached_fwd(q, cache, alpha, f, W, positions.cuda(), seqs=seqs.cuda(),
                          out=torch.full_like(got[0], 3.0), lse=torch.full_like(got[1], 3.0), **opts)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("N,H,Hkv", [(1, 8, 8), (40, 4, 4), (3000, 2, 1), (700, 40, 2)])
def test_cached_default_sequences_and_scale(N, H, Hkv):
    lengths = [1 + (i * 37) % 90 for i in range(N)]
    cache, g = filled(lengths, 8, Hkv, F32, N)
    positions = torch.tensor(lengths).int() - 1
    q = torch.randn(N, H, D, generator=g).cuda()
    f = fa.base("fib", 9)
    got = fa.cached_fwd(q, cache, 0.9, f, 4, positions.cuda(), scale=0.31)
    few = list(range(0, N, max(1, N // 60)))
    part = [t[few] for t in got]
    want = Model(cache).attention(q[few], positions[few], few, slots_of(4, 0.9, f), scale=float(np.float32(0.31)))
    check(part, want, 4, 9)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("W", [8, 25, 90])
@pytest.mark.parametrize("H,Hkv", [(8, 8), (8, 2), (6, 3), (20, 2)])
def test_a_token_by_itself_and_in_a_batch(H, Hkv, W, dtype):
    """The same bits, whatever batch a token is in."""
    cache, g = filled([300, 77, 12], 16, Hkv, dtype, 2)
    N = 2500
    seqs = torch.randint(0, 3, (N,), generator=g).int().cuda()
    positions = (torch.rand(N, generator=g).cuda() * torch.tensor([300, 77, 12]).cuda()[seqs.long()]).int()
    q = tokens(g, N, H, dtype)
    out, lse = fa.cached_fwd(q, cache, 0.8, FIB, W, positions, seqs=seqs)
    for some in (slice(7, 8), slice(100, 400)):
        few = fa.cached_fwd(q[some], cache, 0.8, FIB, W, positions[some].clone(), seqs=seqs[some].clone())
        assert torch.equal(few[0], out[some]) and torch.equal(few[1], lse[some])
    at = torch.randperm(N, generator=g)[:20]
    want = Model(cache).attention(q[at.cuda()], positions.cpu()[at], seqs.cpu()[at], slots_of(W, 0.8, FIB))
    check((out[at.cuda()], lse[at.cuda()]), want, W, len(FIB))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_extreme_scores(dtype):
    """Scores of thousands, apart by more than any exponent, and equal ones."""
    cache, g = filled([50, 50], 16, 1, dtype, 3)
    q = torch.randn(2, 2, D, generator=g) * torch.tensor([[[400.0]], [[0.0]]])
    q = q.to(dtype).cuda()
    positions, seqs = torch.tensor([49, 49]).int(), torch.tensor([0, 1]).int()
    got = fa.cached_fwd(q, cache, 0.8, FIB, 8, positions.cuda(), seqs=seqs.cuda())
    check(got, Model(cache).attention(q, positions, seqs, slots_of(8, 0.8, FIB)), 8, 15)


@pytest.mark.gpu
def test_values_that_are_not_finite():
    """An infinite key of weight 0 and one of all the weight; NaN stays in its head and token."""
    cache, g = filled([20], 32, 2, F32, 5)
    page = int(cache.block_table[0, 0])
    q = torch.ones(2, 2, D).cuda()
    pos, seqs = torch.tensor([19, 8]).int().cuda(), torch.zeros(2, dtype=torch.int32).cuda()
    before = fa.cached_fwd(q, cache, 1.0, [], 4, pos, seqs=seqs)
    cache.v_pages[page, 17, 1] = float("nan")
    out, lse = fa.cached_fwd(q, cache, 1.0, [], 4, pos, seqs=seqs)
    assert torch.isnan(out[0, 1]).all() and torch.equal(lse, before[1])
    assert torch.equal(out[1], before[0][1]) and torch.equal(out[0, 0], before[0][0, 0])
    cache.v_pages[page, 17, 1] = 1.0
    cache.k_pages[page, 18, 0] = 0.0
    cache.k_pages[page, 18, 0, 0] = float("-inf")
    rot = rotated(q.cpu(), pos.cpu())[0, 0, 0]
    out, lse = fa.cached_fwd(q, cache, 1.0, [], 4, pos, seqs=seqs)
    if rot > 0:                                                              # the score is -inf: the row counts for nothing
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    cache.k_pages[page, 15:20, 0] = cache.k_pages[page, 18, 0].clone()
    out, lse = fa.cached_fwd(q, cache, 1.0, [], 4, pos, seqs=seqs)
    if rot > 0:                                                              # nothing is left: 0 / 0
        assert torch.isnan(out[0, 0]).all() and lse[0, 0] == -math.inf
    assert torch.isfinite(out[0, 1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("W", [4, 40])
@pytest.mark.parametrize("N,H,Hkv", [(3, 8, 8), (300, 8, 8), (1100, 8, 8), (1500, 8, 4), (1500, 6, 3), (700, 22, 2)])
def test_values_that_are_not_finite_stay_with_their_heads(N, H, Hkv, W, dtype):
    cache, g = filled([60], 64, Hkv, dtype, 5)
    page = int(cache.block_table[0, 0])
    q = tokens(g, N, H, dtype)
    pos, seqs = torch.full((N,), 19 if W == 4 else 56, dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    before = fa.cached_fwd(q, cache, 1.0, [], W, pos, seqs=seqs)
    for pool, value in ((cache.v_pages, "nan"), (cache.v_pages, "inf"), (cache.k_pages, "nan"), (cache.k_pages, "inf")):
        kept = pool[page, 17, 1].clone()
        pool[page, 17, 1, 3] = float(value)
        out, lse = fa.cached_fwd(q, cache, 1.0, [], W, pos, seqs=seqs)
        pool[page, 17, 1] = kept
        others = [h for h in range(H) if h // (H // Hkv) != 1]
        assert torch.equal(out[:, others], before[0][:, others]) and torch.equal(lse[:, others], before[1][:, others])
        mine = out[:, H // Hkv:2 * H // Hkv]
        if pool is cache.v_pages:
            assert not torch.isfinite(mine[..., 3]).any() and torch.equal(lse, before[1])
        elif value == "nan":
            assert torch.isnan(mine).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("W", [4, 90])
@pytest.mark.parametrize("N,H,Hkv", [(3, 8, 8), (1100, 8, 8), (1500, 8, 2), (700, 22, 2)])
def test_infinite_keys(N, H, Hkv, W, dtype):
    """A score of -infinity leaves its slot out, in a window or a rung; one that is +infinity
    or none makes the output of its token and head NaN, whatever q's roundings are."""
    cache, g = filled([200], 256, Hkv, dtype, 5)
    page = int(cache.block_table[0, 0])
    f = [W + 6.5, W + 16.0]
    slots = slots_of(W, 1.0, f)
    pos, seqs = torch.full((N,), 190).int(), torch.zeros(N).int()
    q = tokens(g, N, H, dtype)
    turned = rotated(q.cpu(), pos)
    few = list(range(0, N, max(1, N // 40)))
    for distance, gone in ((0, 0), (2, 2), (W + 6, W + 1), (W + 7, W + 1), (W + 16, W + 2)):
        left = [s for i, s in enumerate(slots) if i != gone]
        want = Model(cache).attention(q[few], pos[few], seqs[few], left)
        kept = cache.k_pages[page, 190 - distance].clone()
        key = torch.randn(Hkv, D, generator=g)
        key[:, 7], key[::2, 40] = -math.inf, math.inf
        cache.k_pages[page, 190 - distance] = key.to(cache.k_pages.dtype)
        out, lse = fa.cached_fwd(q, cache, 1.0, f, W, pos.cuda(), seqs=seqs.cuda())
        cache.k_pages[page, 190 - distance] = kept
        score = (turned * key.repeat_interleave(H // Hkv, 0)).sum(-1)
        dropped = score == -math.inf
        assert dropped.any() and (~dropped).any() and not torch.isfinite(score).any()
        assert torch.isnan(out.cpu()[~dropped]).all() and not torch.isfinite(lse.cpu()[~dropped]).any()
        at = dropped[few]
        part = [t.cpu()[few].where(at if t.dim() == 2 else at[..., None], w.to(t.dtype)) for t, w in zip((out, lse), want)]
        check(part, want, W, len(f))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_keys_alone(dtype):
    """Nothing is left: 0 / 0, and a sum of nothing."""
    cache, g = filled([1], 16, 2, dtype, 5)
    page = int(cache.block_table[0, 0])
    cache.k_pages[page, 0, 0, 3] = -math.inf
    q = tokens(g, 1, 16, dtype)
    out, lse = fa.cached_fwd(q, cache, 1.0, FIB, 8, torch.zeros(1, dtype=torch.int32, device="cuda"))
    dropped = q[0, :8, 3] > 0                                                # (position 0: q as it is)
    assert dropped.any() and torch.isnan(out[0, :8]).all()
    assert (lse[0, :8][dropped] == -math.inf).all() and not torch.isfinite(lse[0, :8]).any()
    assert torch.isfinite(out[0, 8:]).all() and torch.isfinite(lse[0, 8:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("outlier", [2.0 ** 12, 2.0 ** 20, 2.0 ** 28])
def test_an_outlier_in_a_query(outlier, dtype):
    """One pair of q's dims far above the others, where the keys are 0: the others keep their
    bits.  bf16: q's halves keep 22 bits down to 2^-29 of a head's largest value and all but
    2^-50 of that below it: at most 2^-21.9 of a key here, which the 96 u A of `check` allow
    where sum |q k| is above 2^-4.5 sum |k| (of 62 normal values each: about 2^-0.3)."""
    H = 8
    cache, g = filled([400], 16, H, dtype, 4)
    N = 64
    pos, seqs = torch.randint(0, 400, (N,), generator=g).int(), torch.zeros(N).int()
    q = tokens(g, N, H, dtype).clone()
    cache.k_pages.mul_(8.0)
    for h in range(H):
        m = 4 * h + 1
        cache.k_pages[..., h, m] = cache.k_pages[..., h, m + 32] = 0
        q[:, h, m], q[:, h, m + 32] = outlier, -outlier / 3
    got = fa.cached_fwd(q, cache, 0.8, FIB, 8, pos.cuda(), seqs=seqs.cuda())
    check(got, Model(cache).attention(q, pos, seqs, slots_of(8, 0.8, FIB)), 8, 15)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("W", [8, 90])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_lse_anywhere(offset, W, dtype):
    """lse may be a part of a larger tensor, at any offset; what is beside it stays."""
    cache, g = filled([30, 120], 16, 2, dtype, 2)
    pos, q = torch.tensor([29, 119]).int().cuda(), tokens(g, 2, 4, dtype)
    want = fa.cached_fwd(q, cache, 0.8, FIB, W, pos)
    whole = torch.full((16,), 5.0, device="cuda")
    lse = whole[offset:offset + 8].view(2, 4)
    _, z = fa.cached_fwd(q, cache, 0.8, FIB, W, pos, lse=lse)
    assert z is lse and torch.equal(lse, want[1]) and (whole[:offset] == 5).all() and (whole[offset + 8:] == 5).all()
    whole.fill_(5.0)
    roots = torch.full((2,), -1, dtype=torch.int32, device="cuda")
    fa.tree_fwd(q, cache, 0.8, FIB, W, pos, roots, pos, lse=lse)
    assert torch.equal(lse, want[1]) and (whole[:offset] == 5).all() and (whole[offset + 8:] == 5).all()


@pytest.mark.gpu
def test_what_does_not_exist_is_not_read():
    lengths = [30, 30, 30, 30]
    cache, g = filled(lengths, 8, 2, BF, 8)
    q = tokens(g, 8, 4, BF)
    good = torch.tensor([29, 29, 29, 29]).int()
    seqs = torch.tensor([0, 1, 2, 3]).int()
    want = fa.cached_fwd(q[:4], cache, 0.8, FIB, 8, good.cuda(), seqs=seqs.cuda())
    clear()
    cache.block_table[1, 2] = 10 ** 6                                        # slots 16 .. 23 of sequence 1
    cache.block_table[2, 0] = -1                                             # slots 0 .. 7 of sequence 2, read by rungs
    pos = torch.tensor([29, 29, 29, 29, 2000, 29, 2 ** 31 - 1, 31]).int()    # beyond the table; its own page is not one
    of = torch.tensor([0, 1, 2, 3, 0, 4, 1, 2 ** 31 - 1]).int()
    out, lse = fa.cached_fwd(q, cache, 0.8, FIB, 8, pos.cuda(), seqs=of.cuda())
    with pytest.raises(fa.FibattnError, match="cache does not have|not have") as e:
        fa.check_status()
    assert e.value.flags == 8 and e.value.status == 5
    for n in (0, 3):
        assert torch.equal(out[n], want[0][n]) and torch.equal(lse[n], want[1][n])
    for n in (1, 2, 4, 5, 6, 7):
        assert torch.isnan(out[n]).all() and torch.isnan(lse[n]).all()
    # a page that a query does not reach does not matter: 29 back from 29 is out of W + rungs' rows
    near, _ = fa.cached_fwd(q[:4], cache, 1.0, [], 4, good.cuda(), seqs=seqs.cuda())
    assert torch.isfinite(near).all() and fa.check_status() == 0
    # an append leaves such tokens out
    k = torch.ones(3, 2, D, dtype=BF, device="cuda")
    before = cache.k_pages.clone(), cache.v_pages.clone()
    fa.cache_append(cache, k, k, torch.tensor([3, 16, 5000]).int().cuda(), seqs=torch.tensor([4, 1, 0]).int().cuda())
    with pytest.raises(fa.FibattnError):
        fa.check_status()
    for old, new in zip(before, (cache.k_pages, cache.v_pages)):
        assert torch.equal(old.view(torch.int16), new.view(torch.int16))


# -------------------------------------------------------------------- trees ----

def drafted(g, lengths, sizes, chain=0.9, wide=6):
    """Trees of drafts behind `lengths` cached tokens: seqs, positions, slots, parents."""
    seqs, positions, slots, parents = [], [], [], []
    for b, (have, m) in enumerate(zip(lengths, sizes)):
        first, depth = len(seqs), []
        for t in range(m):
            root = t == 0 or float(torch.rand((), generator=g)) > chain
            up = -1 if root else int(torch.randint(max(0, t - wide), t, (), generator=g))
            depth.append(0 if up < 0 else depth[up] + 1)
            parents.append(up if up < 0 else first + up)
            seqs.append(b)
            positions.append(have + depth[t])
            slots.append(have + t)
    return (torch.tensor(x, dtype=torch.int32) for x in (seqs, positions, slots, parents))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("which", ["usual", "one key", "every rung", "rungs alone", "wide window", "40 rows", "near rungs"])
@pytest.mark.parametrize("H,Hkv,rows,wide", [(1, 1, 1, 3), (8, 2, 16, 6), (6, 3, 13, 1), (3, 3, 100, 70)])
def test_tree(H, Hkv, rows, wide, which, dtype):
    """Trees of 1 to 150 drafts behind 0 to 700 tokens: bushy ones and chains (wide = 1)."""
    W, alpha, f, opts = SETS[which]
    lengths, sizes = [0, 5, 700, 33, 0, 64], [1, 9, 40, 150, 33, 32]
    cache, g = filled(lengths, rows, Hkv, dtype, wide, more=max(sizes))
    seqs, positions, slots, parents = drafted(g, lengths, sizes, 0.97 if wide == 1 else 0.9, wide)
    i32 = [t.cuda() for t in (positions, parents, slots, seqs)]
    k, v = (tokens(g, len(seqs), Hkv, dtype, 1) for _ in range(2))
    fa.cache_append(cache, k, v, i32[0], seqs=i32[3], slots=i32[2])
    q = tokens(g, len(seqs), H, dtype, 2)
    got = fa.tree_fwd(q, cache, alpha, f, W, *i32[:3], seqs=i32[3], **opts)
    want = Model(cache).attention(q, positions, seqs, slots_of(W, alpha, f, **opts), parents=parents, at=slots)
    check(got, want, W, len(f))
    assert fa.check_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("W", [8, 20])
@pytest.mark.parametrize("H,Hkv", [(8, 2), (3, 3), (8, 8), (22, 2)])
def test_many_trees_and_few(H, Hkv, W, dtype):
    """2500 drafts, where a warp takes several key/value heads (bf16) or query heads (fp32):
    the definition, and the same bits as a few sequences at a time; a value that is not
    finite stays with its head."""
    lengths = [(37 * b) % 900 for b in range(50)]
    cache, g = filled(lengths, 16, Hkv, dtype, W, more=50)
    seqs, positions, slots, parents = drafted(g, lengths, [50] * 50)
    i32 = [t.cuda() for t in (positions, parents, slots, seqs)]
    k, v = (tokens(g, 2500, Hkv, dtype, 1) for _ in range(2))
    fa.cache_append(cache, k, v, i32[0], seqs=i32[3], slots=i32[2])
    q = tokens(g, 2500, H, dtype, 2)
    out, lse = fa.tree_fwd(q, cache, 0.8, FIB, W, *i32[:3], seqs=i32[3])
    for b, m in ((0, 1), (7, 3), (48, 2)):                                   # sequences b .. b + m - 1
        at = slice(50 * b, 50 * (b + m))
        up = torch.where(i32[1][at] < 0, -1, i32[1][at] - 50 * b)
        few = fa.tree_fwd(q[at], cache, 0.8, FIB, W, i32[0][at], up, i32[2][at], seqs=i32[3][at])
        assert torch.equal(few[0], out[at]) and torch.equal(few[1], lse[at])
        want = Model(cache).attention(q[at], positions[at], seqs[at], slots_of(W, 0.8, FIB), parents=up.cpu(), at=slots[at])
        check((out[at], lse[at]), want, W, len(FIB))
    page = int(cache.block_table[7, int(slots[350]) // 16])                  # of a root that others read
    cache.v_pages[page, int(slots[350]) % 16, 1, 3] = float("nan")
    again, z = fa.tree_fwd(q, cache, 0.8, FIB, W, *i32[:3], seqs=i32[3])
    mine = torch.arange(H) // (H // Hkv) == 1
    hit = torch.isnan(again[:, mine]).any(-1).any(-1).cpu()
    assert hit[350] and hit.sum() > 1 and (seqs[hit] == 7).all() and torch.equal(z, lse)
    assert torch.equal(again[:, ~mine], out[:, ~mine]) and torch.equal(again[~hit], out[~hit])
    assert fa.check_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_chain_of_drafts_is_the_sequence(dtype):
    """A chain of 100 drafts at their positions' slots, verified, is what cached_fwd computes."""
    cache, g = filled([400], 16, 2, dtype, 1)
    n = 100
    positions = torch.arange(300, 400).int().cuda()
    seqs = torch.zeros(n, dtype=torch.int32).cuda()
    parents = (torch.arange(n) - 1).int().cuda()
    q = tokens(g, n, 4, dtype)
    a = fa.cached_fwd(q, cache, 0.8, FIB, 8, positions, seqs=seqs)
    b = fa.tree_fwd(q, cache, 0.8, FIB, 8, positions, parents, positions, seqs=seqs)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.gpu
def test_drafts_beyond_the_slots_of_positions():
    """Positions may pass the sequence's slots: drafts lie where there is room, and rungs
    reach from there to the sequence's beginning."""
    rows, have = 8, 31                                                       # 4 pages, 32 slots
    table = torch.arange(4, dtype=torch.int32).view(1, 4).cuda()
    cache = fa.PagedCache(*pools("plain", 4, rows, 1, F32), table)
    g = torch.Generator().manual_seed(2)
    put = torch.arange(have).int().cuda()
    zero = torch.zeros(40, dtype=torch.int32).cuda()
    k, v = (torch.randn(40, 1, D, generator=g).cuda() for _ in range(2))
    fa.cache_append(cache, k[:have], v[:have], put, seqs=zero[:have])
    # 9 drafts in the slots 31, 0 .. 7 (whose tokens no draft of this set reads but for the rungs' rows)
    positions = torch.arange(31, 40).int()
    slots = torch.tensor([31, 0, 1, 2, 3, 4, 5, 6, 7]).int()
    parents = (torch.arange(9) - 1).int()
    fa.cache_append(cache, k[have:], v[have:], positions.cuda(), seqs=zero[:9], slots=slots.cuda())
    q = torch.randn(9, 1, D, generator=g).cuda()
    f = [24.0, 31.0, 36.0]
    got = fa.tree_fwd(q, cache, 1.0, f, 3, positions.cuda(), parents.cuda(), slots.cuda(), seqs=zero[:9])
    want = Model(cache).attention(q, positions, torch.zeros(9), slots_of(3, 1.0, f), parents=parents, at=slots)
    check(got, want, 3, 3)


@pytest.mark.gpu
def test_parents_that_do_not_exist():
    cache, g = filled([20, 20], 8, 1, BF, 4, more=8)
    q = tokens(g, 6, 2, BF)
    parents = torch.tensor([-1, 1, 5, -2, 2 ** 31 - 1, 0]).int()             # itself, a later one, ...
    positions = torch.tensor([20, 21, 21, 21, 21, 21]).int()
    slots = torch.arange(20, 26).int()
    seqs = torch.zeros(6, dtype=torch.int32)
    k, v = tokens(g, 6, 1, BF), tokens(g, 6, 1, BF)
    fa.cache_append(cache, k, v, positions.cuda(), seqs=seqs.cuda(), slots=slots.cuda())
    clear()
    out, lse = fa.tree_fwd(q, cache, 0.8, FIB, 8, positions.cuda(), parents.cuda(), slots.cuda(), seqs=seqs.cuda())
    with pytest.raises(fa.FibattnError) as e:
        fa.check_status()
    assert e.value.flags == 8
    bad = torch.tensor([False, True, True, True, True, False])
    assert torch.equal(torch.isnan(out).all(2).all(1).cpu(), bad) and torch.equal(torch.isnan(lse).all(1).cpu(), bad)
    slots[5] = 5000                                                          # a draft's slot that does not exist
    out, _ = fa.tree_fwd(q, cache, 0.8, FIB, 8, positions.cuda(), parents.cuda(), slots.cuda(), seqs=seqs.cuda())
    clear()
    assert torch.isnan(out[5]).all() and torch.isfinite(out[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_parents_elsewhere(dtype):
    """A parent of another sequence, at another position, or that is padding."""
    cache, g = filled([20, 20], 8, 1, dtype, 4, more=8)
    seqs = torch.tensor([0, 1, 0, 0, 0, -1, 0, 0]).int()
    positions = torch.tensor([20, 20, 21, 21, 22, 21, 22, 22]).int()
    parents = torch.tensor([-1, -1, 1, 0, 0, 0, 5, 3]).int()     # 2: of sequence 1; 4: skips one; 6: of padding
    slots = torch.tensor([20, 20, 21, 22, 23, 24, 25, 26]).int()
    q, k, v = tokens(g, 8, 2, dtype), tokens(g, 8, 1, dtype), tokens(g, 8, 1, dtype)
    fa.cache_append(cache, k, v, positions.cuda(), seqs=seqs.cuda(), slots=slots.cuda())
    clear()
    args = [t.cuda() for t in (positions, parents, slots)]
    out, lse = fa.tree_fwd(q, cache, 0.8, FIB, 8, *args, seqs=seqs.cuda())
    with pytest.raises(fa.FibattnError) as e:
        fa.check_status()
    assert e.value.flags == 8
    bad = torch.tensor([False, False, True, False, True, False, True, False])
    assert torch.equal(torch.isnan(out).all(2).all(1).cpu(), bad) and torch.equal(torch.isnan(lse).all(1).cpu(), bad)
    assert not out[5].any()
    # an ancestor that is not read does not matter: the token alone
    out, lse = fa.tree_fwd(q, cache, 1.0, [], 0, *args, seqs=seqs.cuda())
    assert torch.isfinite(out).all() and fa.check_status() == 0


# ------------------------------------------------------------ run together ----

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_generation_agrees_with_the_forward(dtype):
    """Prompts in chunks, then single tokens, then a verified draft: each token's output is
    what `fwd` computes for the whole sequence, as far as both may be from the definition:
    fwd by the tolerances of its own tests, the cache by half a step of its outputs and of
    its fp16 keys, whose scores are then off by 2^-11 of sum |q d k d| <= |q| |k|."""
    g = torch.Generator().manual_seed(6)
    Bn, H, Hkv, T, W, alpha, f = 2, 4, 2, 230, 8, 0.8, fa.base("fib", 15)
    q, k, v = (torch.randn(Bn, h, T, D, generator=g).to(dtype).cuda() for h in (H, Hkv, Hkv))
    out, lse = fa.fwd(q, k, v, alpha, f, W)
    table = torch.randperm(2 * 8, generator=g).int().view(2, 8).cuda()
    cache = fa.PagedCache.empty(16, 32, Hkv, table, dtype=dtype)
    at = 0
    for n in [100, 1, 60, 1, 1, 1, 60, 6]:
        seqs = torch.arange(2).repeat_interleave(n).int().cuda()
        positions = torch.arange(at, at + n).repeat(2).int().cuda()
        qt, kt, vt = (t[:, :, at:at + n].transpose(1, 2).reshape(Bn * n, -1, D) for t in (q, k, v))
        fa.cache_append(cache, kt, vt, positions, seqs=seqs)
        if n == 6:
            parents = (torch.arange(12) - 1).int().cuda()
            parents[6] = -1
            o, z = fa.tree_fwd(qt, cache, alpha, f, W, positions, parents, positions, seqs=seqs)
        else:
            o, z = fa.cached_fwd(qt, cache, alpha, f, W, positions, seqs=seqs)
        want = out[:, :, at:at + n].transpose(1, 2).reshape(Bn * n, H, D).double()
        key = torch.finfo(KEYS[dtype]).eps / 2 * float(q.float().norm(dim=-1).max() * k.float().norm(dim=-1).max()) / 8
        near = torch.finfo(dtype).eps / 2 * want.abs() + 2 * key * float(v.float().abs().max())
        fwd_out = torch.from_numpy(bf16_out_tol(want.cpu().numpy())).cuda() if dtype == BF else 1e-4
        assert ((o.double() - want).abs() <= near * 1.01 + fwd_out + 1e-5).all()
        diff = (z - lse[:, :, at:at + n].transpose(1, 2).reshape(Bn * n, H)).abs().max()
        assert diff <= key + TOL[dtype]["lse"] + 1e-5
        at += n
    assert at == T and fa.check_status() == 0


@pytest.mark.gpu
def test_captured_and_replayed():
    """One graph of append, attention and drafts, replayed as positions and pages change;
    a second graph of the same cache between its replays."""
    cache, g = filled([40, 7, 90], 16, 2, BF, 9, more=40)
    pos = torch.tensor([40, 7, 90]).int().cuda()
    q, k, v = tokens(g, 3, 4, BF, 2), tokens(g, 3, 2, BF), tokens(g, 3, 2, BF)
    roots, slots = torch.full((3,), -1, dtype=torch.int32, device="cuda"), pos.clone()

    def step():
        fa.cache_append(cache, k, v, pos)
        return (*fa.cached_fwd(q, cache, 0.8, FIB, 8, pos), *fa.tree_fwd(q, cache, 0.8, FIB, 8, pos, roots, slots))

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, step()))
        graphs[-1] = (graph, graphs[-1][1])
    for i in range(4):
        for graph, got in graphs:
            pos += 1
            slots.copy_(pos)
            k.copy_(torch.randn(3, 2, D, generator=g))
            if i == 2:                                                       # pages move
                cache.k_pages.copy_(cache.k_pages.flip(0))
                cache.v_pages.copy_(cache.v_pages.flip(0))
                cache.block_table.copy_(torch.where(cache.block_table >= 0, len(cache.k_pages) - 1 - cache.block_table, -1))
            graph.replay()
            want = [t.clone() for t in got]
            assert all(torch.equal(a, b) for a, b in zip(want, step()))
            assert torch.equal(want[0], want[2]) and torch.isfinite(want[0]).all()
    assert fa.check_status() == 0


FIRST = """
import torch, paper_2606_28560_gb300 as fa
table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
pos = torch.arange(30, dtype=torch.int32, device="cuda")
seqs, f = torch.zeros_like(pos), [1.0, 2.0, 3.0, 5.0, 8.0]
for dtype in (torch.bfloat16, torch.float32):
    cache = fa.PagedCache.empty(4, 8, 2, table, dtype=dtype)
    q, k = (torch.randn(30, h, 64, device="cuda").to(dtype) for h in (4, 2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fa.cache_append(cache, k, k, pos, seqs=seqs)
        got = (*fa.cached_fwd(q, cache, 0.8, f, 4, pos, seqs=seqs), *fa.tree_fwd(q, cache, 0.8, f, 4, pos, pos - 1, pos, seqs=seqs))
    graph.replay()
    want = fa.cached_fwd(q, cache, 0.8, f, 4, pos, seqs=seqs)
    assert all(torch.equal(a, b) for a, b in zip(got, (*want, *want))) and fa.check_status() == 0
"""


@pytest.mark.gpu
def test_captured_as_the_first_calls_of_a_program():
    subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, check=True, timeout=300)


@pytest.mark.gpu
def test_on_another_stream():
    """stream=: the arguments are dropped and their memory is asked for again while the other stream waits."""
    cache, g = filled([60, 80], 16, 2, BF, 9, more=4)
    pos, q = torch.tensor([60, 80]).int().cuda(), tokens(g, 2, 4, BF)
    k, v = tokens(g, 2, 2, BF), tokens(g, 2, 2, BF)
    fa.cache_append(cache, k, v, pos)
    want = fa.cached_fwd(q, cache, 0.8, FIB, 8, pos)
    for t in (cache.k_pages, cache.v_pages):
        t[int(cache.block_table[0, 60 // 16]), 60 % 16] = 0
        t[int(cache.block_table[1, 80 // 16]), 80 % 16] = 0
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    given = [t.clone() for t in (k, v, pos, q)]
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)
    fa.cache_append(cache, given[0], given[1], given[2], stream=other)
    got = fa.cached_fwd(given[3], cache, 0.8, FIB, 8, given[2], stream=other)
    del given
    for n in {t.numel() * t.element_size() for t in (k, v, pos, q, *want)}:
        junk = [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(8)]
        del junk
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_rows_beyond_32_bits_of_offset():
    """Pages that lie more than 2^32 elements into their pools."""
    pages, rows, Hkv = 560_000, 16, 8                                        # 4.6e9 elements
    table = torch.tensor([[pages - 1, 3, 540_000], [530_000, pages - 2, 0]], dtype=torch.int32).cuda()
    cache = fa.PagedCache(*(torch.empty(pages, rows, Hkv, D, dtype=t, device="cuda") for t in (torch.float16, BF)), table)
    g = torch.Generator().manual_seed(1)
    seqs, positions = torch.arange(2).repeat_interleave(48).int(), torch.arange(48).repeat(2).int()
    k, v, q = tokens(g, 96, Hkv, BF), tokens(g, 96, Hkv, BF), tokens(g, 96, 8, BF)
    fa.cache_append(cache, k, v, positions.cuda(), seqs=seqs.cuda())
    got = fa.cached_fwd(q, cache, 0.8, FIB, 8, positions.cuda(), seqs=seqs.cuda())
    small = fa.PagedCache(cache.k_pages[table.long().flatten()], cache.v_pages[table.long().flatten()],
                          torch.arange(6, dtype=torch.int32).view(2, 3).cuda())
    again = fa.cached_fwd(q, small, 0.8, FIB, 8, positions.cuda(), seqs=seqs.cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    check(got, Model(small).attention(q, positions, seqs, slots_of(8, 0.8, FIB)), 8, 15)


@pytest.mark.gpu
def test_two_streams_at_once():
    """Two sequences of one cache, generated on two streams."""
    cache, g = filled([100, 100], 16, 2, BF, 12, more=30)
    q, k, v = tokens(g, 60, 4, BF), tokens(g, 60, 2, BF), tokens(g, 60, 2, BF)
    pos = [(torch.tensor([100 + i]).int().cuda(), torch.tensor([b]).int().cuda()) for i in range(30) for b in range(2)]
    streams_ = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for n, (p, s) in enumerate(pos):
        fa.cache_append(cache, k[n:n + 1], v[n:n + 1], p, seqs=s, stream=streams_[n % 2])
        outs.append(fa.cached_fwd(q[n:n + 1], cache, 0.8, FIB, 8, p, seqs=s, stream=streams_[n % 2]))
    torch.cuda.synchronize()
    for n, (p, s) in enumerate(pos):
        want = fa.cached_fwd(q[n:n + 1], cache, 0.8, FIB, 8, p, seqs=s)
        assert all(torch.equal(a, b) for a, b in zip(outs[n], want))


# ---------------------------------------------------------- refusals, on CPU ----

def test_struct_is_the_headers(tmp_path):
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include "fibattn.h"\n#include <stddef.h>\nint main(void) { printf("%zu %zu %zu", '
                   'sizeof(fibattn_cache), offsetof(fibattn_cache, ready), offsetof(fibattn_cache, phase)); return 0; }\n')
    exe = tmp_path / "size"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    S = B.CacheStruct
    assert got == f"{ctypes.sizeof(S)} {S.ready.offset} {S.phase.offset}"


def init(c=None, k=256, v=256, pages=4, rows=8, Hkv=2, d=64, ps=1024, rs=128, hs=64, table=256, seqs=3, per=5, dtype=1, base=0.0):
    c = B.CacheStruct() if c is None else c
    rc = B.lib().fibattn_cache_init(ctypes.addressof(c), k, v, pages, rows, Hkv, d, ps, rs, hs, table, seqs, per, dtype, base)
    return c, rc, fa.binding.lib().fibattn_last_error().decode()


@pytest.mark.parametrize("change,status,words", [
    (dict(k=0), 1, "NULL"), (dict(v=0), 1, "NULL"), (dict(table=0), 1, "NULL"), (dict(k=264), 1, "aligned"),
    (dict(table=258), 1, "aligned"), (dict(pages=0), 1, "at least 1"), (dict(rows=0), 1, "at least 1"),
    (dict(Hkv=-1), 1, "at least 1"), (dict(seqs=0), 1, "at least 1"), (dict(per=0), 1, "at least 1"), (dict(d=128), 2, "64"),
    (dict(ps=1000), 1, "multiples of 64"), (dict(rs=0), 1, "multiples of 64"), (dict(hs=-64), 1, "multiples of 64"),
    (dict(ps=1 << 40, pages=2), 1, "2^32"), (dict(ps=1 << 62, pages=2 ** 31 - 1), 1, "2^32"),
    (dict(ps=64 << 16, pages=1 << 17), 1, "2^32"),
    (dict(rows=1 << 16, per=1 << 15), 1, "2^30"), (dict(dtype=7), 1, "dtype"), (dict(base=1.0), 1, "rope_base"),
    (dict(base=float("nan")), 1, "rope_base"), (dict(base=float("inf")), 1, "rope_base"),
])
def test_init_refuses(change, status, words):
    c, rc, _ = init()
    assert rc == 0
    c, rc, message = init(c, **change)
    assert rc == status and words in message
    assert B.lib().fibattn_cache_append(ctypes.addressof(c), 256, 64, 64, 256, 64, 64, 256, None, None, 1, None) == 1
    assert "cache_init" in B.lib().fibattn_last_error().decode()


def append(c, **k):
    a = dict(k=256, kt=128, kh=64, v=256, vt=128, vh=64, positions=256, slots=None, seqs=None, N=1) | k
    rc = B.lib().fibattn_cache_append(c and ctypes.addressof(c), *a.values(), None)
    return rc, B.lib().fibattn_last_error().decode()


@pytest.mark.parametrize("change,words", [
    (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(positions=None), "NULL"), (dict(k=260), "aligned"),
    (dict(v=264), "aligned"), (dict(kt=4), "16 bytes"), (dict(vh=-64), "16 bytes"), (dict(N=-1), "negative"),
    (dict(N=2 ** 30), "2^31"),
])
def test_append_refuses(change, words):
    c, rc, _ = init()
    assert rc == 0
    rc, message = append(c, **change)
    assert rc == 1 and words in message
    assert append(None)[0] == 1 and append(B.CacheStruct())[0] == 1
    assert append(c, N=0, k=None)[0] == 0


def attend(c, tree, opts=None, **k):
    f = np.array([1.0, 2.0, 3.0], dtype=np.float32)
    a = dict(q=256, qt=256, qh=64, out=256, lse=256, positions=256, parents=256, slots=256, seqs=None, N=1, H=4, W=8,
             alpha=1.0, f=f.ctypes.data, K=3) | k
    if not tree:
        del a["parents"], a["slots"]
    call = B.lib().fibattn_tree_fwd if tree else B.lib().fibattn_cached_fwd
    rc = call(c and ctypes.addressof(c), *a.values(), opts and ctypes.addressof(opts), None)
    return rc, B.lib().fibattn_last_error().decode()


@pytest.mark.parametrize("tree", [False, True])
def test_attention_refuses_an_lse_between_values(tree):
    c, _, _ = init()
    rc, message = attend(c, tree, lse=258)
    assert rc == 1 and "lse: 4-byte" in message


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("change,words", [
    (dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(lse=None), "NULL"), (dict(positions=None), "NULL"),
    (dict(q=264), "aligned"), (dict(out=272 + 8), "aligned"), (dict(qt=7), "16 bytes"), (dict(qh=-8), "16 bytes"),
    (dict(N=-1), "negative"), (dict(H=3), "multiple"), (dict(H=0), "multiple"), (dict(N=2 ** 30), "2^31"),
    (dict(W=-1), "W must"), (dict(W=1025), "W must"), (dict(K=33), "K must"), (dict(K=-1), "K must"), (dict(f=None), "offsets"),
    (dict(alpha=0.4), "alpha"), (dict(alpha=float("nan")), "alpha"),
])
def test_attention_refuses(change, words, tree):
    c, rc, _ = init()
    assert rc == 0
    rc, message = attend(c, tree, **change)
    assert rc == 1 and words in message
    assert attend(None, tree)[0] == 1
    assert attend(c, tree, N=0, q=None)[0] == 0
    for field, value in (("rope_base", 1e4), ("Hkv", 2), ("fwd_kernel", 1), ("bwd_kernel", 1), ("rotated_k", 256),
                         ("residuals", 256)):
        o = B.Opts()
        setattr(o, field, value)
        assert attend(c, tree, o)[0] == 1
    o = B.Opts(scale=float("inf"))
    assert attend(c, tree, o)[0] == 1


@pytest.mark.parametrize("which", ["positions", "slots", "seqs", "parents"])
def test_integers_between_values_are_refused(which):
    c, _, _ = init()
    calls = [(lambda k: attend(c, True, **k))]
    if which != "parents":
        calls.append(lambda k: append(c, **k))
    if which in ("positions", "seqs"):
        calls.append(lambda k: attend(c, False, **k))
    for call in calls:
        for at in (257, 258, 259):
            rc, message = call({which: at})
            assert rc == 1 and "4-byte aligned" in message and which in message


def test_tree_refuses_no_parents():
    c, _, _ = init()
    assert attend(c, True, parents=None)[0] == 1 and attend(c, True, slots=None)[0] == 1


def i32(n, device="cuda:0"):
    return torch.empty(n, dtype=torch.int32, device=device)


def fake_cache(device="cuda:0", dtype=BF, Hkv=2):
    return fa.PagedCache.empty(4, 8, Hkv, torch.empty(3, 5, dtype=torch.int32, device=device), dtype=dtype)


def test_binding_refuses_caches(library):   # noqa: F811
    t = torch.empty(3, 5, dtype=torch.int32, device="cuda:0")

    def pool(*shape, dtype=BF, device="cuda:0"):
        return torch.empty(*(shape or (4, 8, 2, 64)), dtype=dtype, device=device)

    h = torch.float16
    for k, v, table, error in [
            (pool(4, 8, 2, 32, dtype=h), pool(4, 8, 2, 32), t, ValueError), (pool(4, 8, 64, dtype=h), pool(4, 8, 64), t, ValueError),
            (pool(dtype=h), pool(4, 8, 1, 64), t, ValueError), (pool(), pool(), t, TypeError),
            (pool(dtype=h), pool(dtype=F32), t, TypeError), (pool(dtype=h), pool(dtype=h), t, TypeError),
            (pool(dtype=h), pool(device="cuda:1"), t, ValueError), (pool(dtype=h, device="cpu"), pool(device="cpu"), t, ValueError),
            (pool(dtype=h), pool(), t.cpu(), ValueError), (pool(dtype=h), pool(), t.long(), ValueError),
            (pool(dtype=h), pool(), t[0], ValueError), (pool(dtype=h), pool(), t[:, ::2], ValueError),
            (pool(4, 8, 2, 128, dtype=h)[..., ::2], pool(4, 8, 2, 128)[..., ::2], t, ValueError),
            (pool(dtype=h), pool(4, 2, 8, 64).transpose(1, 2), t, ValueError)]:
        with pytest.raises(error):
            fa.PagedCache(k, v, table)
    assert not library.calls
    with pytest.raises(TypeError):
        fa.PagedCache.empty(4, 8, 2, t, dtype=torch.float16)


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "block_table", "rope_base", "dtype", "Hkv", "index", "device"])
def test_a_caches_parts_stay(name, library):   # noqa: F811
    """What the library was told of at the start cannot be replaced behind its back."""
    cache = fake_cache()
    was = {n: getattr(cache, n) for n in ("k_pages", "v_pages", "block_table")}
    with pytest.raises(AttributeError, match="make a new"):
        setattr(cache, name, torch.empty(3, 9, dtype=torch.int32, device="cuda:0"))
    with pytest.raises(AttributeError, match="make a new"):
        delattr(cache, name)
    with pytest.raises(AttributeError, match="make a new"):
        cache.__init__(*was.values())
    assert all(getattr(cache, n) is t for n, t in was.items())
    cache.note = "layer 3"                                                   # a caller's own attribute
    cache.note = "layer 4"
    assert cache.note == "layer 4"
    del cache.note
    assert not hasattr(cache, "note")


@pytest.mark.parametrize("layers", [0, 0.0, 1e4, 10000])
@pytest.mark.parametrize("caches", [0, 0.0, 1e4, 10000])
def test_a_rope_base_of_zero_is_the_librarys_own(layers, caches, library):   # noqa: F811
    """0 and 1e4 are one rotation, as they are for `fwd`: a layer of one takes a cache of the other."""
    layer = fa.FibAttention(rope_base=layers)
    table = torch.empty(3, 5, dtype=torch.int32, device="cuda:0")
    cache = fa.PagedCache.empty(4, 8, 2, table, rope_base=caches)
    q = torch.empty(5, 2, 64, dtype=BF, device="cuda:0")
    library.calls.clear()
    layer.cached(q, cache, i32(5), alpha=1.0)
    assert [name for name, _ in library.calls] == ["fibattn_cached_fwd"]
    with pytest.raises(ValueError, match="rope_base"):
        fa.FibAttention(rope_base=5e5).cached(q, cache, i32(5), alpha=1.0)


def test_binding_refuses_sizes_beyond_an_int(library):   # noqa: F811
    """More than 31 bits would arrive at the library cut short: 2^32 + 1 tokens as one."""
    cache = fake_cache()
    library.calls.clear()
    one, n = torch.empty(1, 2, 64, dtype=BF, device="cuda:0"), 2 ** 32 + 1
    many, p = one.expand(n, 2, 64), i32(n)
    for call in (lambda: fa.cache_append(cache, many, many, p), lambda: fa.cached_fwd(many, cache, 1.0, [1.0], 8, p),
                 lambda: fa.tree_fwd(many, cache, 1.0, [1.0], 8, p, p, p)):
        with pytest.raises(ValueError, match="2.31"):
            call()
    for W in (2 ** 32 + 8, 2 ** 31, -2 ** 32):
        with pytest.raises(ValueError, match="W must"):
            fa.cached_fwd(one, cache, 1.0, [1.0], W, i32(1))
    for table in ((n, 5), (3, n)):
        with pytest.raises(ValueError, match="2.31"):
            fa.PagedCache.empty(4, 8, 2, torch.empty(table, dtype=torch.int32, device="cuda:0"))
    assert not library.calls


def test_binding_refuses_tokens(library):   # noqa: F811
    cache = fake_cache()
    library.calls.clear()
    ok, p = torch.empty(5, 2, 64, dtype=BF, device="cuda:0"), i32(5)
    for k, v, kw in [
            (ok.float(), ok, {}), (ok, ok.float(), {}), (ok[:, :1], ok[:, :1], {}), (ok, ok[:4], {}), (ok[0], ok[0], {}),
            (ok.cpu(), ok, {}), (ok[..., :32], ok, {}), (torch.empty(5, 64, 2, dtype=BF, device="cuda:0").transpose(1, 2), ok, {}),
            (torch.empty(5, 2, 68, dtype=BF, device="cuda:0")[..., :64], ok, {}), (ok, ok, dict(seqs=i32(4))),
            (ok, ok, dict(slots=p.long())), (ok, ok, dict(seqs=i32(5, "cpu"))), (ok, ok, dict(slots=i32(10)[::2]))]:
        with pytest.raises(ValueError):
            fa.cache_append(cache, k, v, p, **kw)
    for bad in (p.long(), i32(4), i32(5, "cuda:1"), None):
        with pytest.raises(ValueError):
            fa.cache_append(cache, ok, ok, bad)
        with pytest.raises(ValueError):
            fa.cached_fwd(ok, cache, 1.0, [1.0], 8, bad)
        with pytest.raises(ValueError):
            fa.tree_fwd(ok, cache, 1.0, [1.0], 8, p, p if bad is None else bad, bad)
    for kw in (dict(out=ok.float()), dict(out=ok[:4]), dict(out=ok.cpu()), dict(lse=torch.empty(5, 2)),
               dict(lse=torch.empty(5, 2, dtype=BF, device="cuda:0")), dict(lse=torch.empty(2, 5, device="cuda:0").t())):
        with pytest.raises(ValueError):
            fa.cached_fwd(ok, cache, 1.0, [1.0], 8, p, **kw)
    other = fake_cache("cuda:1")
    library.calls.clear()
    one = torch.empty(5, 2, 64, dtype=BF, device="cuda:1")
    for call in (lambda: fa.cache_append(other, one, one, i32(5, "cuda:1")),
                 lambda: fa.cached_fwd(one, other, 1.0, [1.0], 8, i32(5, "cuda:1")),
                 lambda: fa.tree_fwd(one, other, 1.0, [1.0], 8, *[i32(5, "cuda:1") for _ in range(3)])):
        with pytest.raises(ValueError, match="current device is cuda:0"):
            call()
    assert not library.calls


@pytest.mark.parametrize("name", ["cache_append", "cached_fwd", "tree_fwd"])
def test_memory_of_a_call_on_another_stream(name, library, streams):   # noqa: F811
    caller, other, allocated, recorded = streams
    cache, x = fake_cache(), torch.empty(5, 2, 64, dtype=BF, device="cuda:0")
    given = [i32(5) for _ in range(4)]
    allocated.clear()
    call = {"cache_append": lambda s: fa.cache_append(cache, x, x, given[0], seqs=given[1], slots=given[2], stream=s),
            "cached_fwd": lambda s: fa.cached_fwd(x, cache, 1.0, [1.0], 8, given[0], seqs=given[1], stream=s),
            "tree_fwd": lambda s: fa.tree_fwd(x, cache, 1.0, [1.0], 8, given[0], given[1], given[2], seqs=given[3], stream=s)}[name]
    library.calls.clear()
    results = call(other) or ()
    (_, args), = library.calls
    assert args[-1] == other.cuda_stream and all(s is other for _, s in allocated)
    used = [cache.k_pages, cache.v_pages, cache.block_table, x] + given[:{"cache_append": 3, "cached_fwd": 2, "tree_fwd": 4}[name]]
    assert all(any(t is r and s is other for r, s in recorded) for t in used)
    assert all(any(t is r and s is caller for r, s in recorded) for t in results)
    recorded.clear()
    call(caller)
    assert not recorded
