"""Linear cross entropy (loss, lse and both gradients) against the definition
in 64 bits, over types, sizes from one row to many, odd and ragged ones, rows
without a target, and refusals.

Tolerances follow from the arithmetic.  With u = 2^-23 (an fp32 sum that may
truncate) and S = max |x| . |w| over the products of a logit, a logit is within
e = (D + 8) u S; lse and loss within 2 e + 16 u (1 + |lse|).  A gradient entry
is a sum of |g| |w| terms, |g| <= dloss (p + onehot): each term is off by 2 e
(through p) and, with bf16 I/O, by the 2^-8 of g's own rounding; the sum adds K u
and the result's rounding 2^-8 (bf16) or u.
"""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2606_28560_gb300 as fa
from paper_2606_28560_gb300 import binding as B
from paper_2606_28560_gb300 import build as build_mod

U = 2.0 ** -23
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(N, D, V, dtype, seed, mask="some", scale=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, D, generator=g)
    w = torch.randn(V, D, generator=g) * (scale / D ** 0.5)
    t = torch.randint(0, V, (N,), generator=g)
    if N:
        t[0], t[-1] = 0, V - 1                    # the first and the last column
    if mask == "some":
        t[torch.rand(N, generator=g) < 0.3] = -100
    elif mask == "all":
        t[:] = -100
    dl = torch.rand(N, generator=g) + 0.1
    return x.to(dtype).cuda(), w.to(dtype).cuda(), t.cuda(), dl.cuda()


def truth(x, w, t, dl):
    """The definition in fp64, and the bounds of the module's docstring."""
    D, V, N = x.shape[1], w.shape[0], x.shape[0]
    x, w, dl = x.double(), w.double(), dl.double()
    s = x @ w.t()
    e = (D + 8) * U * float((x.abs() @ w.abs().t()).max())
    lse = torch.logsumexp(s, 1)
    has = t != -100
    one = torch.zeros_like(s)
    one[has, t[has]] = 1.0
    loss = (lse - (s * one).sum(1)) * has
    p = torch.exp(s - lse[:, None])
    c = (dl * has)[:, None]
    g, a = c * (p - one), c * (p + one)
    return dict(lse=lse, loss=loss, dx=g @ w, dw=g.t() @ x, e=e, tol=2 * e + 16 * U * (1 + lse.abs().max()),
                ax=a @ w.abs(), aw=a.t() @ x.abs())


def check(x, w, t, dl, tag=""):
    r = truth(x, w, t, dl)
    bf = x.dtype == torch.bfloat16
    loss, lse = fa.linear_xent_fwd(x, w, t)
    assert (lse.double() - r["lse"]).abs().max() <= r["tol"], tag
    assert (loss.double() - r["loss"]).abs().max() <= r["tol"], tag
    assert not loss[t == -100].any()
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    for name, got, want, mag, K in (("dx", dx, r["dx"], r["ax"], w.shape[0]), ("dw", dw, r["dw"], r["aw"], x.shape[0])):
        rel = 2 * r["tol"] + (K + 8) * U + (2.0 ** -8 if bf else 0.0)
        tol = rel * mag + (2.0 ** -8 if bf else U) * want.abs() + 1e-30
        bad = (got.double() - want).abs() > tol
        assert not bad.any(), f"{tag} {name}: {int(bad.sum())} of {bad.numel()} beyond the bound"
        norm = float(want.norm())
        if norm > 0:                              # two independent bf16 roundings: 2^-9 sqrt(2/3) = 1.6e-3, twice that at most
            off = float((got.double() - want).norm()) / norm
            assert off <= (3.2e-3 if bf else 1e-5), f"{tag} {name}: {off}"
    assert not dx[t == -100].any()
    return loss, lse, dx, dw


SIZES = [(1, 1, 1), (1, 64, 257), (3, 7, 5), (2, 512, 4096), (100, 64, 257), (129, 100, 1000), (257, 72, 513),
         (256, 64, 256), (255, 128, 255), (1001, 100, 5003), (300, 520, 20011), (64, 2048, 3001), (513, 1030, 700),
         (1024, 512, 2048), (7, 1536, 30000), (2049, 8, 31), (128, 333, 128),
         # one to four rows, few rows, tiles: each border, odd widths, a vocabulary that ends inside a tile
         (4, 2048, 501), (4, 2056, 501), (5, 33, 17), (8, 136, 4099), (9, 512, 1003), (16, 1000, 2001), (17, 130, 999),
         (32, 260, 1234), (33, 260, 1234), (32, 1604, 300), (16, 3205, 70), (8, 6404, 40), (31, 3, 1025)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_matches_definition(size, dtype):
    check(*make(*size, TYPES[dtype], seed=sum(size)))


# two, eight, sixteen and 32 rows on both sides of 2^22 weights, rows of x that fill a
# block's shared memory, small heads that are spread over the processors
HEADS = [(2, 300, 20011), (3, 512, 9000), (4, 512, 9000), (8, 1032, 5001), (9, 1032, 5001), (16, 1024, 5001), (17, 1024, 5001),
         (32, 2044, 3001), (24, 1500, 4099), (32, 512, 8192), (32, 512, 8193), (16, 2048, 17), (12, 1601, 1000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", HEADS, ids=lambda s: "x".join(map(str, s)))
def test_small_batches_over_heads(size, dtype):
    check(*make(*size, TYPES[dtype], seed=sum(size)))


# rows of x deeper than a block's shared memory, and as deep
DEEP = [(8, 7168, 200), (4, 7176, 900), (8, 8192, 333), (12, 7999, 517), (32, 8190, 100), (1, 8192, 50), (16, 3584, 300), (16, 3592, 300),
        (8, 4096, 700)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", DEEP, ids=lambda s: "x".join(map(str, s)))
def test_small_batches_of_deep_rows(size, dtype):
    check(*make(*size, TYPES[dtype], seed=sum(size)))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 9, 32, 100])
@pytest.mark.parametrize("bits", [0x7fc00000, 0x7fffffff, -1, 0x7f800001])
def test_nan_of_any_payload(bits, rows):
    x, w, t, dl = make(rows, 40, 300, torch.float32, 12)
    t[:] = torch.arange(rows, device="cuda")
    x.view(torch.int32)[1, 3] = bits
    loss, lse = fa.linear_xent_fwd(x, w, t)
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    assert torch.isnan(loss[1]) and torch.isnan(lse[1]) and torch.isnan(dx[1]).all() and torch.isnan(dw).all()
    others = torch.arange(rows, device="cuda") != 1
    assert torch.isfinite(loss[others]).all() and torch.isfinite(dx[others]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("mask", ["none", "all"])
def test_masks(mask, dtype):
    x, w, t, dl = make(300, 96, 777, TYPES[dtype], 5, mask)
    loss, lse, dx, dw = check(x, w, t, dl)
    if mask == "all":
        assert not loss.any() and not dx.any() and not dw.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_several_pieces_of_the_vocabulary(dtype):
    # g of all columns is above the piece limit: several pieces, the last one ragged
    check(*make(20000, 72, 20003, TYPES[dtype], 6))


@pytest.mark.gpu
@pytest.mark.parametrize("N", [1, 8, 40])
def test_offsets_beyond_31_bits(N):
    """w and dw of more than 2^31 values: the definition in 64 bits a piece of the vocabulary at a time."""
    D, V, piece = 2056 if N > 1 else 2048, 1_050_000, 1 << 16
    x, w0, _, dl = make(N, D, piece, torch.bfloat16, 13, "none")
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for k, at in enumerate(range(0, V, piece)):
        w[at:at + piece] = w0.roll(k, 0)[:V - at]
    t = V - 1 - 3 * torch.arange(N, device="cuda")
    assert w.numel() > 2 ** 31
    s = torch.cat([x.double() @ w[at:at + piece].double().t() for at in range(0, V, piece)], 1)
    e = (D + 8) * U * float((x.double().abs() @ w0.double().abs().t()).max())      # every piece has w0's rows
    want_lse = torch.logsumexp(s, 1)
    tol = 2 * e + 16 * U * (1 + float(want_lse.abs().max()))
    loss, lse = fa.linear_xent_fwd(x, w, t)
    assert (lse.double() - want_lse).abs().max() <= tol
    assert (loss.double() - (want_lse - s.gather(1, t[:, None])[:, 0])).abs().max() <= tol
    g = torch.exp(s - want_lse[:, None])
    g[torch.arange(N, device="cuda"), t] -= 1.0
    g *= dl.double()[:, None]
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    want_dx, off = 0, 0
    for at in range(0, V, piece):
        part = g[:, at:at + piece]
        want_dx = want_dx + part @ w[at:at + piece].double()
        off += float((dw[at:at + piece].double() - part.t() @ x.double()).square().sum())
    # by norms, with the bound that the whole matrices of the other tests have
    assert float((dx.double() - want_dx).norm()) <= 3.2e-3 * float(want_dx.norm())
    assert off ** 0.5 <= 3.2e-3 * float(sum((g[:, at:at + piece].t() @ x.double()).square().sum() for at in range(0, V, piece))) ** 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_large_logits(dtype):
    # spread of thousands: exp of anything but the maximum vanishes, nothing overflows
    x, w, t, dl = make(130, 64, 1000, TYPES[dtype], 7, scale=2000.0)
    loss, lse, dx, dw = check(x, w, t, dl)
    assert all(torch.isfinite(v).all() for v in (loss, lse, dx, dw))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [64, 65, 520])
@pytest.mark.parametrize("N", [1, 3, 8, 20, 40, 300])
@pytest.mark.parametrize("value", ["lowest", "-inf"])
def test_columns_masked_by_a_bias(value, N, D, dtype):
    """A head with a bias, as a column of w against ones in x.  The bias of tokens
    that are not to be had is the type's lowest value or -infinity: single tokens,
    and a block of the vocabulary.  They add nothing."""
    V, T = 1500, TYPES[dtype]
    x, w, t, dl = make(N, D, V, T, 25, "none")
    out = torch.zeros(V, dtype=torch.bool, device="cuda")
    out[::3] = True
    out[200:1200] = True
    left = (~out).nonzero()[:, 0]
    t = torch.where(out[t], left[t % len(left)], t)
    t[-1] = V - 1 if not out[V - 1] else V - 2
    x[:, -1], w[:, -1] = 1.0, 0.0
    w[out, -1] = torch.finfo(T).min if value == "lowest" else -float("inf")
    at = torch.searchsorted(left, t)
    r = truth(x, w[left], at, dl)
    loss, lse = fa.linear_xent_fwd(x, w, t)
    assert (lse.double() - r["lse"]).abs().max() <= r["tol"] and (loss.double() - r["loss"]).abs().max() <= r["tol"]
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    bf = dtype == "bf16"
    assert not dw[out].any()
    for got, want, mag, K in ((dx[:, :-1], r["dx"][:, :-1], r["ax"][:, :-1], V), (dw[left], r["dw"], r["aw"], N)):
        rel = 2 * r["tol"] + (K + 8) * U + (2.0 ** -8 if bf else 0.0)
        assert ((got.double() - want).abs() <= rel * mag + (2.0 ** -8 if bf else U) * want.abs() + 1e-30).all()
    if value == "lowest":                         # (0 times an infinity is none, as in any matrix product)
        assert not dx[:, -1].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [64, 520])
@pytest.mark.parametrize("N", [2, 20, 40, 300])
def test_rows_with_nothing_but_masked_columns(N, D, dtype):
    """All logits are the type's lowest value (what x and w have besides vanishes
    beside it): equal logits, next to which log V vanishes too."""
    V, T = 600, TYPES[dtype]
    x, w, t, dl = make(N, D, V, T, 26, "none")
    low = torch.finfo(T).min
    x[:, -1], w[:, -1] = 1.0, low
    loss, lse = fa.linear_xent_fwd(x, w, t)
    assert ((lse.double() - low).abs() <= (D + 8) * U * abs(low)).all() and (loss == 0).all()
    dw = fa.linear_xent_bwd(x, w, t, lse, dl)[1]
    # exp(s - lse) is 1 there, as in the plain form: g = dloss (1 - [v = target])
    one = torch.nn.functional.one_hot(t, V).double()
    want = (dl.double()[:, None] * (1 - one)).t() @ x.double()
    assert float((dw.double() - want).norm()) <= 3.2e-3 * float(want.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_zero_rows_and_columns(dtype):
    x, w, t, dl = make(200, 64, 300, TYPES[dtype], 8)
    x[5], w[:] = 0, w
    w[17] = 0
    check(x, w, t, dl)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_row_that_is_not_finite_stays_alone(value, dtype):
    x, w, t, dl = make(200, 64, 300, TYPES[dtype], 9, "none")
    clean, _ = fa.linear_xent_fwd(x, w, t)
    lse0 = fa.linear_xent_fwd(x, w, t)[1]
    dx0, _ = fa.linear_xent_bwd(x, w, t, lse0, dl)
    x[37, 3] = value
    loss, lse = fa.linear_xent_fwd(x, w, t)
    keep = torch.arange(200, device="cuda") != 37
    assert torch.equal(loss[keep], clean[keep]) and not torch.isfinite(loss[37])
    dx, _ = fa.linear_xent_bwd(x, w, t, lse, dl)
    assert torch.equal(dx[keep], dx0[keep])
    t[37] = -100                                  # without a target: loss and dx are exactly zero
    loss, lse = fa.linear_xent_fwd(x, w, t)
    dx, _ = fa.linear_xent_bwd(x, w, t, lse, dl)
    assert loss[37] == 0 and not dx[37].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_target_outside_the_vocabulary(dtype):
    x, w, t, dl = make(150, 64, 300, TYPES[dtype], 10, "none")
    fa.check_status()
    want = t.clone()
    want[[3, 140, 149]] = -100
    t[3], t[140], t[149] = 300, -1, 2 ** 40
    loss, lse = fa.linear_xent_fwd(x, w, t)
    with pytest.raises(fa.FibattnError) as ei:
        fa.check_status()
    assert ei.value.status == 5 and ei.value.flags == 4
    assert torch.isnan(loss[[3, 140, 149]]).all() and int(torch.isnan(loss).sum()) == 3
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    with pytest.raises(fa.FibattnError):
        fa.check_status()
    dx2, dw2 = fa.linear_xent_bwd(x, w, want, lse, dl)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    assert fa.check_status() == 0


@pytest.mark.gpu
def test_other_ignore_index():
    x, w, t, dl = make(90, 64, 200, torch.bfloat16, 11)
    t2 = torch.where(t == -100, torch.full_like(t, 7), torch.where(t == 7, torch.full_like(t, 8), t))
    want = torch.where(t2 == 7, torch.full_like(t, -100), t2)
    a, b = fa.linear_xent_fwd(x, w, t2, ignore_index=7), fa.linear_xent_fwd(x, w, want)
    assert torch.equal(a[0], b[0])
    g, h = fa.linear_xent_bwd(x, w, t2, a[1], dl, ignore_index=7), fa.linear_xent_bwd(x, w, want, b[1], dl)
    assert torch.equal(g[0], h[0]) and torch.equal(g[1], h[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_no_rows(dtype):
    x, w, t, dl = make(0, 64, 300, TYPES[dtype], 12)
    loss, lse = fa.linear_xent_fwd(x, w, t)
    assert loss.shape == (0,)
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    assert dx.shape == (0, 64) and not dw.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_same_result_every_time_and_on_another_stream(dtype):
    x, w, t, dl = make(700, 200, 9001, TYPES[dtype], 13)
    first = fa.linear_xent_fwd(x, w, t)
    first += fa.linear_xent_bwd(x, w, t, first[1], dl)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s):
            again = fa.linear_xent_fwd(x, w, t)
            again += fa.linear_xent_bwd(x, w, t, again[1], dl)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [2, 300])
def test_in_a_captured_graph(N, dtype):
    """Replays on changed inputs give what direct calls give."""
    x, w, t, dl = make(N, 136, 2000, TYPES[dtype], 19)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):                    # warm up off the capture
        loss, lse = fa.linear_xent_fwd(x, w, t)
        fa.linear_xent_bwd(x, w, t, lse, dl)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss, lse = fa.linear_xent_fwd(x, w, t)
        dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    x2, w2, t2, dl2 = make(N, 136, 2000, TYPES[dtype], 20)
    for a, b in ((x, x2), (w, w2), (t, t2), (dl, dl2)):
        a.copy_(b)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    want = fa.linear_xent_fwd(x2, w2, t2)
    want += fa.linear_xent_bwd(x2, w2, t2, want[1], dl2)
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), want))


@pytest.mark.gpu
def test_depth_beyond_a_run_of_the_tensor_core():
    """Positive operands, whose truncated sums would drift if a deep logit were
    summed by the tensor core alone (128 steps of 16 at some 2e-8 each: 3e-6 of a
    sum of some hundreds, 1e-3).  Runs of 512 keep the drift below 32 steps'."""
    g = torch.Generator().manual_seed(21)
    x, w = (torch.rand(n, 2048, generator=g).bfloat16().cuda() for n in (300, 700))
    w /= 8
    t = torch.randint(0, 700, (300,), generator=g).cuda()
    s = x.double() @ w.double().t()
    lse = fa.linear_xent_fwd(x, w, t)[1]
    off = (lse.double() - torch.logsumexp(s, 1)).abs().max()
    # 32 steps of 2^-24 to 2^-23 of a run's sum (a quarter of s), four runs, their fp32 sums, lse's own rounding
    assert float(off) <= float(s.abs().max()) * (32 * 2.0 ** -23 + 8 * 2.0 ** -24)


@pytest.mark.gpu
def test_depth_of_the_products_beyond_a_run():
    """dw over 2^18 rows, all terms positive: what truncation takes from a sum grows
    with the depth that the tensor core sums alone, by 2.2e-8 (sums 512 deep) to
    4.3e-8 (4096 deep) of the sum for each 16.  Runs of 2^17 keep it below
    2^13 * 4.3e-8; the roundings of g and of dw go both ways and leave the median."""
    N, D, V = 1 << 18, 8192, 1024
    g = torch.Generator(device="cuda").manual_seed(22)
    x = torch.rand(N, D, generator=g, device="cuda", dtype=torch.bfloat16).add_(0.5)
    w = (torch.randn(V, D, generator=g, device="cuda") * 0.038).bfloat16()
    t = torch.zeros(N, dtype=torch.int64, device="cuda")
    dl = torch.rand(N, generator=g, device="cuda") * 0.5 + 0.5
    lse = fa.linear_xent_fwd(x, w, t)[1]
    dw = fa.linear_xent_bwd(x, w, t, lse, dl)[1]
    some = torch.arange(7, V, 32, device="cuda")
    want = torch.zeros(len(some), D, dtype=torch.float64, device="cuda")
    for at in range(0, N, 1 << 14):
        rows = slice(at, at + (1 << 14))
        xd = x[rows].double()
        want += (torch.exp(xd @ w[some].double().t() - lse[rows, None].double()) * dl[rows, None]).t() @ xd
    off = float(((dw[some].double() - want) / want).median())
    assert abs(off) <= 2 ** 13 * 4.3e-8, off


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_millions_of_rows(dtype):
    # more rows than g of 256 columns fits in 512 MiB
    check(*make((1 << 21) + 5, 8, 520, TYPES[dtype], 24))


# deep products over tiles of one block and of two, whole and cut, with a ragged last run
@pytest.mark.gpu
@pytest.mark.parametrize("size", [(70_001, 300, 515), (33_000, 1030, 700), (100_000, 100, 300), (300, 520, 70_001), (270, 2056, 40_000),
                                  (40_000, 2100, 2000)], ids=lambda s: "x".join(map(str, s)))
def test_products_in_several_runs(size):
    check(*make(*size, torch.bfloat16, seed=sum(size)))


@pytest.mark.gpu
def test_pieces_of_a_vocabulary_above_2_18():
    check(*make(2100, 264, 270_001, torch.bfloat16, 23))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_writes_only_its_outputs(dtype):
    """Outputs and workspace lie between guards of a known pattern."""
    N, D, V = 130, 72, 515
    x, w, t, dl = make(N, D, V, TYPES[dtype], 14)

    def guarded(nbytes):
        pad = 4096
        buf = torch.full((pad + (nbytes + 255) // 256 * 256 + pad,), 0x5a, dtype=torch.uint8, device="cuda")
        return buf, buf[pad:pad + nbytes]

    code = B._dtype_code(x)
    es = x.element_size()
    sizes = dict(loss=N * 4, lse=N * 4, dx=N * D * es, dw=V * D * es,
                 wf=B.lib().fibattn_linear_xent_fwd_workspace_bytes(N, D, V, code),
                 wb=B.lib().fibattn_linear_xent_bwd_workspace_bytes(N, D, V, code))
    bufs = {k: guarded(v) for k, v in sizes.items()}
    v = {k: b[1] for k, b in bufs.items()}
    loss, lse = fa.linear_xent_fwd(x, w, t, loss=v["loss"].view(torch.float32), lse=v["lse"].view(torch.float32),
                                   workspace=v["wf"])
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl, dx=v["dx"].view(x.dtype).view(N, D), dw=v["dw"].view(x.dtype).view(V, D),
                                workspace=v["wb"])
    torch.cuda.synchronize()
    for k, (buf, _) in bufs.items():
        n = sizes[k]
        assert bool((buf[:4096] == 0x5a).all()) and bool((buf[4096 + n:] == 0x5a).all()), k
    plain = fa.linear_xent_fwd(x, w, t)
    assert torch.equal(plain[0], loss) and torch.equal(plain[1], lse)
    g = fa.linear_xent_bwd(x, w, t, lse, dl)
    assert torch.equal(g[0], dx) and torch.equal(g[1], dw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [0, 3, 700])
def test_one_gradient_alone(N, dtype):
    x, w, t, dl = make(N, 520, 1500, TYPES[dtype], 18)
    _, lse = fa.linear_xent_fwd(x, w, t)
    dx, dw = fa.linear_xent_bwd(x, w, t, lse, dl)
    a, none = fa.linear_xent_bwd(x, w, t, lse, dl, want_dw=False)
    none2, b = fa.linear_xent_bwd(x, w, t, lse, dl, want_dx=False)
    assert none is None and none2 is None
    # the depth may be cut elsewhere: the sums' roundings, and bf16's own
    for got, want in ((a, dx), (b, dw)):
        if want.numel():
            tol = (2.0 ** -8 if dtype == "bf16" else 4e-6) * max(1e-30, float(want.double().norm()))
            assert float((got.double() - want.double()).norm()) <= tol
    x.requires_grad_(True)                        # a frozen head
    if N:
        fa.linear_cross_entropy(x, w, t).backward()
        assert x.grad is not None and w.grad is None


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the library's own loss; a loss is within some 1e-6 in
    fp32, so a quotient over 2 h = 0.04 is within 1e-4, plus h^2 of the third derivative."""
    x, w, t, dl = make(5, 6, 7, torch.float32, 15, "none")
    t[2] = -100
    h = 0.02

    def total(x, w):
        return float((fa.linear_xent_fwd(x, w, t)[0].double() * dl.double()).sum())

    _, lse = fa.linear_xent_fwd(x, w, t)
    grads = fa.linear_xent_bwd(x, w, t, lse, dl)
    for which, g in enumerate(grads):
        for i in range(g.shape[0]):
            for j in range(g.shape[1]):
                at = []
                for sign in (1, -1):
                    y = [x.clone(), w.clone()]
                    y[which][i, j] += sign * h
                    at.append(total(*y))
                assert abs((at[0] - at[1]) / (2 * h) - float(g[i, j])) <= 2e-3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd(reduction, dtype):
    x, w, t, _ = make(60, 64, 131, TYPES[dtype], 16)
    x, t = x.view(3, 20, 64), t.view(3, 20)
    x.requires_grad_(True)
    w.requires_grad_(True)
    loss = fa.linear_cross_entropy(x, w, t, reduction=reduction)
    up = torch.rand(loss.shape, device="cuda") + 0.5
    (loss * up).sum().backward()
    has = (t != -100).view(-1)
    dl = {"mean": (up / has.sum()).expand(60), "sum": up.expand(60), "none": up.reshape(-1)}[reduction] if \
        reduction != "none" else up.reshape(-1)
    r = truth(x.detach().view(60, 64), w.detach(), t.view(-1), dl.contiguous())
    want = {"mean": r["loss"].sum() / has.sum(), "sum": r["loss"].sum(), "none": r["loss"].view(3, 20)}[reduction]
    assert (loss.double() - want).abs().max() <= (1 if reduction != "sum" else 60) * r["tol"] + 64 * U * want.abs().max()
    bf = dtype == "bf16"
    for got, ref in ((x.grad.view(60, 64), r["dx"]), (w.grad, r["dw"])):
        assert float((got.double() - ref).norm() / ref.norm()) <= (3.2e-3 if bf else 1e-5)


# -------------------------------------------------------------- refusals ----

@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def _fwd(x=256, w=256, t=256, loss=256, lse=256, N=4, D=8, V=16, dtype=1, ws=256, nbytes=1 << 30):
    vp = ctypes.c_void_p
    return B.lib().fibattn_linear_xent_fwd(vp(x), vp(w), vp(t), vp(loss), vp(lse), N, D, V, -100, dtype, vp(ws), nbytes,
                                           None)


def _bwd(x=256, w=256, t=256, lse=256, dl=256, dx=256, dw=256, N=4, D=8, V=16, dtype=1, ws=256, nbytes=1 << 30):
    vp = ctypes.c_void_p
    return B.lib().fibattn_linear_xent_bwd(vp(x), vp(w), vp(t), vp(lse), vp(dl), vp(dx), vp(dw), N, D, V, -100, dtype,
                                           vp(ws), nbytes, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("bad", [dict(N=-1), dict(N=(1 << 24) + 1), dict(D=0), dict(D=8193), dict(V=0),
                                 dict(V=(1 << 24) + 1), dict(dtype=2), dict(x=0), dict(w=0), dict(t=0), dict(lse=0),
                                 dict(ws=0), dict(x=264), dict(w=257), dict(t=260), dict(lse=260), dict(ws=264),
                                 dict(nbytes=16)], ids=str)
def test_refused_before_any_launch(call, bad):
    assert call(**bad) == 1
    assert B.lib().fibattn_last_error()


def test_refused_outputs():
    assert _fwd(loss=0) == 1 and _fwd(loss=264) == 1
    assert _bwd(dl=0) == 1 and _bwd(dx=0, dw=0) == 1
    for name in ("dl", "dx", "dw"):
        assert _bwd(**{name: 264}) == 1


def test_no_rows_need_no_pointers():
    assert _fwd(0, 0, 0, 0, 0, N=0, ws=0, nbytes=0) == 0


def test_workspace_sizes():
    f, b = B.lib().fibattn_linear_xent_fwd_workspace_bytes, B.lib().fibattn_linear_xent_bwd_workspace_bytes
    assert f(-1, 64, 100, 1) == 0 and b(4, 0, 100, 1) == 0 and b(4, 64, 100, 7) == 0
    # far below the fp32 logits of the same call
    assert 0 < f(16384, 512, 32768, 1) < 16384 * 32768 * 4 // 64
    assert 0 < b(16384, 512, 32768, 1) < 16384 * 32768 * 4 // 3


MIB = 1 << 20


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [40, 20_000, 1 << 20, 1 << 21, 1 << 24])
def test_workspace_of_many_rows(N, dtype):
    """What the header says of g: 512 MiB or 256 columns, whichever is more.  The
    rest: both operands as planes, dx over the pieces, sums over a part of a depth."""
    D, V, code, planes = 64, 32768, list(TYPES).index(dtype), 3 if dtype == "f32" else 1
    need = B.lib().fibattn_linear_xent_bwd_workspace_bytes(N, D, V, code)
    g = 2 * planes * N * V
    if g > 512 * MIB:
        g = max(512 * MIB, 256 * 2 * planes * N)
    rest = (2 * planes * (N + V) * D if dtype == "f32" else 0) + 4 * N * D
    assert g * 0.99 <= need <= g + rest + 128 * MIB


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,rows", [(3, 8), (8, 8), (9, 16), (17, 32), (32, 32)])
def test_workspace_of_few_rows(N, rows, dtype):
    """g of all columns in fp32, where the call is one of few rows."""
    D, V = 64, 1 << 24
    need = B.lib().fibattn_linear_xent_bwd_workspace_bytes(N, D, V, list(TYPES).index(dtype))
    few = dtype == "f32" or N <= 16                # bf16 over a large head, D <= 1024
    g = 4 * rows * V if few else 512 * MIB
    assert g * 0.99 <= need <= g + (1 << 30 if not few else 64 * MIB)


def test_python_checks():
    x, w, t = torch.zeros(4, 8), torch.zeros(16, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        fa.linear_xent_fwd(x, w, t)
    with pytest.raises(ValueError, match=r"\[N, D\]"):
        fa.linear_xent_fwd(x, w[:, :4], t)
    with pytest.raises(ValueError, match=r"\[N, D\]"):
        fa.linear_xent_fwd(x, w, t[:3])
    with pytest.raises(ValueError, match="reduction"):
        fa.linear_cross_entropy(x, w, t, reduction="max")
    with pytest.raises(ValueError, match="targets"):
        fa.linear_cross_entropy(x, w, t.view(2, 2))


@pytest.mark.gpu
def test_python_checks_on_tensors():
    x, w, t, dl = make(8, 16, 20, torch.bfloat16, 17)
    with pytest.raises(ValueError, match="contiguous"):
        fa.linear_xent_fwd(x.t().contiguous().t(), w, t)
    with pytest.raises(ValueError, match="one dtype"):
        fa.linear_xent_fwd(x, w.float(), t)
    with pytest.raises(TypeError):
        fa.linear_xent_fwd(x.half(), w.half(), t)
    with pytest.raises(ValueError, match="int64"):
        fa.linear_xent_fwd(x, w, t.int())
    _, lse = fa.linear_xent_fwd(x, w, t)
    with pytest.raises(ValueError, match="dloss"):
        fa.linear_xent_bwd(x, w, t, lse, dl.double())
    with pytest.raises(ValueError, match="lse"):
        fa.linear_xent_bwd(x, w, t, lse[:4], dl)
    with pytest.raises(ValueError, match="dx and dw"):
        fa.linear_xent_bwd(x, w, t, lse, dl, dx=x.float())
    with pytest.raises(fa.FibattnError, match="aligned"):
        flat = torch.zeros(8 * 16 + 1, dtype=torch.bfloat16, device="cuda")
        fa.linear_xent_fwd(flat[1:].view(8, 16), w, t)
    with pytest.raises(fa.FibattnError, match="workspace"):
        fa.linear_xent_fwd(x, w, t, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
