"""Global gradient norm and clipping against the definition in 64 bits, over
types, sizes from nothing to more than a block's, views at odd offsets, many
tensors, norms that are not finite, and refusals.

Tolerances: squares are summed in fp32 over at most 256 values and in fp64
beyond, so the sum is within 258 * 2^-24 of itself and norm within half that
and its own rounding; an output adds the rounding of the coefficient and its own
(2^-9 in bf16, taken twice for values that fall between).
"""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2606_28560_gb300 as fa
from paper_2606_28560_gb300 import binding as B
from paper_2606_28560_gb300 import build as build_mod

NORM_TOL = 131 * 2.0 ** -24
OUT_TOL = {torch.float32: NORM_TOL + 2.0 ** -22, torch.bfloat16: 2.0 ** -8}
GUARD = 16
PATTERN = 0.34375                                 # exact in both types


def tensors(spec, seed, offset=0, scale=1.0):
    """[(size, dtype)] as views between guards of one flat buffer per tensor."""
    g = torch.Generator().manual_seed(seed)
    views, flats = [], []
    for k, (n, dtype) in enumerate(spec):
        at = GUARD + (offset * (k + 1)) % 8
        flat = torch.full((at + n + GUARD,), PATTERN, dtype=dtype, device="cuda")
        flat[at:at + n] = (torch.randn(n, generator=g) * scale).to(dtype).cuda()
        views.append(flat[at:at + n])
        flats.append((flat, at, n))
    return views, flats


def guards_hold(flats):
    return all(bool((f[:a] == PATTERN).all()) and bool((f[a + n:] == PATTERN).all()) for f, a, n in flats)


def truth(grads, max_norm):
    norm = math.sqrt(sum(float(t.double().pow(2).sum()) for t in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def close(got, src, coef):
    for o, s in zip(got, src):
        want = s.double() * coef
        assert ((o.double() - want).abs() <= OUT_TOL[s.dtype] * want.abs() + 1e-37).all()


F, H = torch.float32, torch.bfloat16
SPECS = {
    "one value": [(1, F)], "one bf16 value": [(1, H)], "nothing": [(0, F), (0, H)],
    "nothing between": [(5, F), (0, F), (7, H), (0, H), (3, F)],
    "small mix": [(1, F), (64, H), (4096, H), (63, F), (1, F), (257 * 64, H)],
    "around a chunk": [(16383, F), (16384, F), (16385, F), (16383, H), (16384, H), (16385, H), (32769, H)],
    "one large": [(5_000_003, H)], "large f32": [(3_000_001, F), (1, F), (2_000_000, F)],
    "many": [((k * 37) % 300, F if k % 3 else H) for k in range(1300)],
}


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1, 3, 4])
@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0])
@pytest.mark.parametrize("spec", list(SPECS))
def test_matches_definition(spec, max_norm, offset):
    grads, gflats = tensors(SPECS[spec], len(spec), offset)
    outs, oflats = tensors([(n, d) for n, d in SPECS[spec]], 1, offset + 2)      # other alignment than the gradients
    keep = [g.clone() for g in grads]
    want, coef = truth(grads, max_norm)
    norm = fa.clip_grads(grads, max_norm, out=outs)
    assert abs(float(norm) - want) <= NORM_TOL * want
    close(outs, keep, coef)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep)) and guards_hold(gflats) and guards_hold(oflats)
    if coef == 1.0:
        assert all(torch.equal(a, b) for a, b in zip(outs, keep))
    alone = fa.grad_norm(grads)
    assert torch.equal(alone, norm) and all(torch.equal(a, b) for a, b in zip(grads, keep))
    placed = fa.clip_grads(grads, max_norm)                                      # in place
    assert torch.equal(placed, norm) and guards_hold(gflats)
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.gpu
def test_no_tensors():
    assert float(fa.clip_grads([], 1.0)) == 0.0 and float(fa.grad_norm([])) == 0.0
    assert float(fa.clip_grad_norm_([torch.nn.Parameter(torch.zeros(3, device="cuda"))], 1.0)) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F, H])
def test_not_finite(dtype):
    for value in (float("nan"), float("inf")):
        a = torch.ones(40000, dtype=dtype, device="cuda")
        b = torch.ones(7, dtype=dtype, device="cuda")
        a[30001] = value
        norm = fa.clip_grads([a, b], 1.0)
        if math.isnan(value):
            assert math.isnan(float(norm)) and bool(torch.isnan(a).all()) and bool(torch.isnan(b).all())
        else:                                     # the formula: coefficient 0, and 0 * inf
            assert math.isinf(float(norm)) and not b.any()
            assert bool(torch.isnan(a[30001])) and int(torch.isnan(a).sum()) == 1


@pytest.mark.gpu
def test_unlimited():
    a = torch.randn(1000, device="cuda")
    keep = a.clone()
    norm = fa.clip_grads([a], float("inf"))
    assert torch.equal(a, keep) and abs(float(norm) - float(keep.double().norm())) <= NORM_TOL * float(norm)


@pytest.mark.gpu
def test_more_than_31_bits_of_bytes():
    """A tensor whose byte offsets pass 2^31 and 2^32."""
    n = (1 << 31) + 5
    a = torch.zeros(n, dtype=H, device="cuda")
    a[n - 1] = 3.0
    a[(1 << 30) + 1] = 4.0
    norm = fa.clip_grads([a], 1.0)
    assert abs(float(norm) - 5.0) <= 5.0 * NORM_TOL
    want = torch.tensor([3.0, 4.0], dtype=torch.float64) / (5.0 + 1e-6)
    got = torch.stack([a[n - 1], a[(1 << 30) + 1]]).double().cpu()
    assert ((got - want).abs() <= OUT_TOL[H] * want).all() and int(torch.count_nonzero(a)) == 2


@pytest.mark.gpu
def test_same_result_every_time_and_on_another_stream():
    grads, _ = tensors(SPECS["around a chunk"] + SPECS["large f32"], 3, 1)
    first = fa.grad_norm(grads)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(s):
            again = fa.grad_norm(grads)
        s.synchronize()
        assert torch.equal(first, again)


@pytest.mark.gpu
def test_in_a_captured_graph():
    grads, _ = tensors(SPECS["small mix"] + SPECS["around a chunk"], 5, 1)
    outs, _ = tensors(SPECS["small mix"] + SPECS["around a chunk"], 6, 3)
    fa.clip_grads(grads, 1.0, out=outs)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        norm = fa.clip_grads(grads, 1.0, out=outs)
    for t in grads:
        t.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    want, coef = truth(grads, 1.0)
    assert abs(float(norm) - want) <= NORM_TOL * want
    close(outs, grads, coef)


@pytest.mark.gpu
def test_parameters():
    m = torch.nn.Sequential(torch.nn.Linear(33, 65), torch.nn.Linear(65, 9), torch.nn.Linear(9, 1)).cuda()
    m[2].weight.requires_grad_(False)             # a parameter without a gradient
    (m(torch.randn(50, 33, device="cuda")).square().sum() * 100).backward()
    keep = [p.grad.clone() for p in m.parameters() if p.grad is not None]
    want, coef = truth(keep, 1.0)
    norm = fa.clip_grad_norm_(m.parameters(), 1.0)
    assert abs(float(norm) - want) <= NORM_TOL * want and coef < 1
    close([p.grad for p in m.parameters() if p.grad is not None], keep, coef)
    assert m[2].weight.grad is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("scale", [1e20, 1e30, 1e-18, 1e-24, 1e-34])
@pytest.mark.parametrize("offset", [0, 3])
def test_values_whose_squares_leave_fp32(offset, scale, dtype):
    """The norm of finite values is theirs, and large ones are clipped to it, though
    no square of theirs is an fp32 number.  1e-18: squares are numbers, sums of a
    thread lie below the limit of the second way."""
    grads, flats = tensors([(n, dtype) for n in (1, 7, 4099, 70001)], 9, offset, scale)
    keep = [g.clone() for g in grads]
    want, coef = truth(grads, 1.0)
    norm = fa.clip_grads(grads, 1.0)
    assert abs(float(norm) - want) <= NORM_TOL * want and guards_hold(flats)
    close(grads, keep, coef)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("at", [0, 1, 8, 2047, 40000, 69999, 70000])
def test_one_large_value_among_ordinary_ones(at, dtype):
    a = torch.randn(70001, generator=torch.Generator().manual_seed(at)).to(dtype).cuda()
    a[at] = 3e25
    keep, (want, coef) = a.clone(), truth([a], 1.0)
    norm = fa.clip_grads([a], 1.0)
    assert abs(float(norm) - want) <= NORM_TOL * want
    close([a], [keep], coef)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F, H])
def test_zeros_with_a_tiny_value(dtype):
    a = torch.zeros(200_000, dtype=dtype, device="cuda")
    a[::2] = -0.0
    assert float(fa.grad_norm([a])) == 0.0
    a[123_457] = 2.0 ** -100
    assert float(fa.grad_norm([a])) == 2.0 ** -100


# -------------------------------------------------------------- refusals ----

@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def _call(n=1, grads=(256,), outs=(256,), sizes=(4,), types=(0,), max_norm=1.0, norm=256, ws=256, nbytes=1 << 20):
    vp = ctypes.c_void_p
    g = (vp * max(1, len(grads)))(*grads) if grads is not None else None
    o = (vp * max(1, len(outs)))(*outs) if outs is not None else None
    return B.lib().fibattn_clip_grads(n, g, o, (ctypes.c_longlong * len(sizes))(*sizes), (ctypes.c_int * len(types))(*types),
                                      max_norm, vp(norm), vp(ws), nbytes, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=(1 << 20) + 1), dict(grads=None), dict(norm=0), dict(ws=0),
                                 dict(norm=258), dict(ws=264), dict(max_norm=-1.0), dict(max_norm=float("nan")),
                                 dict(nbytes=8), dict(types=(2,)), dict(sizes=(-1,)), dict(grads=(0,)), dict(outs=(0,)),
                                 dict(grads=(258,)), dict(outs=(257,)), dict(sizes=(1 << 62,))], ids=str)
def test_refused_before_any_launch(bad):
    assert _call(**bad) == 1
    assert B.lib().fibattn_last_error()


def test_python_checks():
    with pytest.raises(ValueError, match="CUDA"):
        fa.clip_grads([torch.zeros(3)], 1.0)
    with pytest.raises(TypeError):
        fa.clip_grads([torch.zeros(3, dtype=torch.float16)], 1.0)
    with pytest.raises(ValueError, match="one tensor for each"):
        fa.clip_grads([torch.zeros(3)], 1.0, out=[])


@pytest.mark.gpu
def test_python_checks_on_tensors():
    a = torch.zeros(4, 4, device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        fa.clip_grads([a.t()], 1.0)
    with pytest.raises(ValueError, match="like the gradients"):
        fa.clip_grads([a], 1.0, out=[a.bfloat16()])
    with pytest.raises(ValueError, match="like the gradients"):
        fa.clip_grads([a], 1.0, out=[a[:2]])
    with pytest.raises(fa.FibattnError, match="max_norm"):
        fa.clip_grads([a], -1.0)
