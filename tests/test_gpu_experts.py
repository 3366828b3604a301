"""The operators of a layer of experts on the GPU against plain implementations in 64 bits.

Tolerances.  u = 2^-24 is the rounding of one fp32 operation.  A sum of n fp32 terms in any order is within n * u of the
sum of the terms' magnitudes; what is rounded to an output type is within half a step of it.  Scores: the exponential's
argument x - max is rounded once (|x - max| < 128, so 2^7 * u) and the exponential, the sum of at most 1024 (37 additions
deep in the warp) and the quotient add less than 50 u: 2^8 * u = 1.6e-5 relative covers a score and a renormalised weight.
"""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SCORE_TOL = 2.0 ** 8 * U
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}
SMALLEST = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -130, torch.float16: 2.0 ** -25}      # half the smallest step of the type
FMAX = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _close(got, want, bound):
    """|got - want| <= bound everywhere (fp64)."""
    got, want = got.double(), want.double()
    off = (got - want).abs() - bound
    assert not torch.isnan(got).any()
    assert float(off.max() if off.numel() else -1.0) <= 0.0, float(off.max())


# ---------------------------------------------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------------------------------------------

def _scores64(x, score):
    x = x.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    m = x.amax(1, keepdim=True)
    e = torch.where(x == m, torch.ones_like(x), torch.exp(x - m))
    return e / e.sum(1, keepdim=True)


def _route64(x, top_k, score, bias, groups, kept, group_top):
    """ids, chosen scores, and per token whether every decision is clear of rounding."""
    p = _scores64(x, score).cpu()
    x = x.double().cpu()
    by_logit = bias is None and group_top == 1
    key = x if by_logit else p + (0 if bias is None else bias.double().cpu())
    T, E = x.shape
    per = E // groups
    ids, chosen, clear = torch.full((T, top_k), -1, dtype=torch.int64), torch.zeros(T, top_k, dtype=torch.float64), torch.ones(T, dtype=torch.bool)
    gap = 0.0 if by_logit else 1e-5
    for t in range(T):
        there = [e for e in range(E) if x[t, e] > -math.inf and key[t, e] > -math.inf]
        if kept < groups:
            of = []
            for g in range(groups):
                best = sorted((float(key[t, e]) for e in there if e // per == g), reverse=True)[:group_top]
                of.append(sum(best) if best else -math.inf)
            order = sorted((g for g in range(groups) if of[g] > -math.inf), key=lambda g: (-of[g], g))
            if len(order) > kept and of[order[kept - 1]] - of[order[kept]] < gap:
                clear[t] = False
            there = [e for e in there if e // per in order[:kept]]
        there.sort(key=lambda e: (-float(key[t, e]), e))
        for a, b in zip(there[:top_k], there[1:top_k + 1]):
            if float(key[t, a]) - float(key[t, b]) < gap:
                clear[t] = False
        for j, e in enumerate(there[:top_k]):
            ids[t, j], chosen[t, j] = e, p[t, e]
    return ids, chosen, clear


def _check_plan(ids, E, align, offsets, rows, source):
    ids, offsets, rows, source = (v.cpu().tolist() for v in (ids, offsets, rows, source))
    flat = [e for r in ids for e in r]
    want_rows, want_source, at = [-1] * len(flat), [-1] * len(source), 0
    for e in range(E):
        assert offsets[e] == at
        n = 0
        for i, v in enumerate(flat):
            if v == e:
                want_rows[i], want_source[at + n] = at + n, i
                n += 1
        at += -(-n // align) * align
    assert offsets[E] == at
    assert [r for v in rows for r in v] == want_rows
    assert source == want_source


def _route_check(x, top_k, *, score="softmax", bias=None, groups=1, kept=1, group_top=1, renormalise=True, scale=1.0, align=1, min_clear=0.9):
    ids, w, offsets, rows, source = pkg.asgd_route(x, top_k, score=score, bias=bias, groups=groups, groups_kept=kept, group_top=group_top,
                                                   renormalise=renormalise, scale=scale, align=align)
    want, chosen, clear = _route64(x, top_k, score, bias, groups, kept, group_top)
    assert clear.double().mean() >= min_clear
    assert torch.equal(ids.cpu().long()[clear], want[clear])
    ww = scale * chosen / (chosen.sum(1, keepdim=True) + 1e-20) if renormalise else scale * chosen
    _close(w.cpu()[clear], ww[clear], 2 * SCORE_TOL * ww[clear].abs() + 1e-30)
    _check_plan(ids, x.shape[1], align, offsets, rows, source)
    return ids, w


@pytest.mark.parametrize("T, E, top_k, score, groups, kept, group_top, dtype, align, biased", [
    (1, 1, 1, "softmax", 1, 1, 1, F32, 1, False),
    (1, 256, 8, "sigmoid", 8, 4, 2, BF, 1, True),
    (3, 7, 7, "softmax", 1, 1, 1, F16, 1, False),
    (64, 60, 6, "sigmoid", 4, 3, 2, F32, 128, True),
    (65, 60, 6, "sigmoid", 4, 3, 1, F32, 16, True),
    (333, 128, 8, "softmax", 1, 1, 1, BF, 128, False),
    (200, 96, 4, "softmax", 6, 2, 1, F16, 1, False),
    (130, 96, 4, "softmax", 3, 2, 2, F32, 7, True),
    (129, 32, 32, "sigmoid", 1, 1, 1, F32, 1, True),
    (70, 1000, 32, "softmax", 1, 1, 1, F32, 4, False),
    (40, 1024, 5, "sigmoid", 32, 3, 2, BF, 1, True),
    (190, 512, 10, "sigmoid", 16, 16, 2, F32, 1, False),
])
def test_route(T, E, top_k, score, groups, kept, group_top, dtype, align, biased):
    g = _gen(T * 1000 + E)
    x = (torch.randn(T, E, generator=g, device="cuda") * 2).to(dtype)
    bias = torch.randn(E, generator=g, device="cuda") * 0.2 if biased else None
    for renormalise, scale in ((True, 2.5), (False, 1.0)):
        # among many experts near ties are frequent
        _route_check(x, top_k, score=score, bias=bias, groups=groups, kept=kept, group_top=group_top, renormalise=renormalise, scale=scale,
                     align=align, min_clear=0.5 if E >= 512 or dtype != F32 else 0.9)


def test_route_without_plan_and_without_tokens():
    x = torch.randn(50, 40, device="cuda")
    ids, w = pkg.asgd_route(x, 3, plan=False)
    full = pkg.asgd_route(x, 3)
    assert torch.equal(ids, full[0]) and torch.equal(w, full[1])
    ids, w, offsets, rows, source = pkg.asgd_route(x[:0], 3, align=8)
    assert ids.shape == (0, 3) and w.shape == (0, 3) and rows.shape == (0, 3)
    assert not offsets.any() and torch.equal(source, torch.full((40 * 7,), -1, dtype=torch.int32, device="cuda"))


def test_route_ties_go_to_the_lowest_index():
    x = torch.randint(0, 3, (300, 64), generator=_gen(5), device="cuda").float()
    x[0] = 0.0
    x[1] = -0.0
    x[1, 5] = 0.0                                        # the zeros of both signs are equal
    _route_check(x, 8, min_clear=1.0)
    _route_check(x, 8, groups=8, kept=3, min_clear=1.0)
    ids, _ = pkg.asgd_route(x, 8, score="sigmoid", bias=torch.zeros(64, device="cuda"), plan=False)
    assert torch.equal(ids, pkg.asgd_route(x, 8, score="sigmoid", plan=False)[0])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_route_masks(score, dtype):
    E, lowest = 48, torch.finfo(dtype).min
    x = torch.randn(140, E, generator=_gen(7), device="cuda").to(dtype)
    x[0] = -math.inf                                     # nothing is available
    x[1] = -math.inf
    x[1, 17] = 1.0                                       # one expert is
    x[2, 5:] = -math.inf
    x[3] = lowest                                        # the type's lowest value is a number
    x[4, 3:] = lowest
    x[5] = -math.inf
    x[5, [3, 30]] = lowest
    x[70:] = torch.where(torch.rand(70, E, generator=_gen(8), device="cuda") < 0.8, torch.full((), -math.inf, device="cuda", dtype=dtype), x[70:])
    ids, w = _route_check(x, 6, score=score, align=4, min_clear=1.0)
    assert (ids[0] == -1).all() and (w[0] == 0).all()
    assert ids[1].tolist() == [17, -1, -1, -1, -1, -1]
    assert not torch.isnan(w).any()
    bias = torch.zeros(E, device="cuda")
    bias[::2] = -math.inf                                # a bias takes experts out as well
    ids, _ = _route_check(x.float(), 6, score=score, bias=bias, min_clear=0.3)
    assert ((ids % 2 == 1) | (ids == -1)).all()


def test_route_nan_and_infinity():
    x = torch.randn(100, 40, generator=_gen(9), device="cuda")
    clean = pkg.asgd_route(x, 4, plan=False)
    y = x.clone()
    y[10, 3] = math.nan
    y[11] = math.nan
    y[12, [4, 9]] = math.inf
    for score in ("softmax", "sigmoid"):
        ids, w, offsets, rows, source = pkg.asgd_route(y, 4, score=score, align=8)
        _check_plan(ids, 40, 8, offsets, rows, source)
        assert 3 not in ids[10].tolist() and (ids[11] == -1).all() and sorted(ids[12, :2].tolist()) == [4, 9]
        assert torch.isfinite(w[12]).all() and (w[11] == 0).all()
        if score == "softmax":
            assert torch.isnan(w[10]).all() and w[12].tolist() == [0.5, 0.5, 0.0, 0.0]
            keep = [t for t in range(100) if t not in (10, 11, 12)]
            assert torch.equal(ids[keep], clean[0][keep]) and torch.equal(w[keep], clean[1][keep])


def test_route_strides_streams_and_repeats():
    big = torch.randn(500, 90, generator=_gen(11), device="cuda")
    x = big[:, 7:71]                                     # rows 90 apart, no 16-byte alignment
    want = pkg.asgd_route(x.contiguous(), 5, align=128)
    for got in (pkg.asgd_route(x, 5, align=128), pkg.asgd_route(x, 5, align=128)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.asgd_route(x, 5, align=128, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_route_plan_over_many_chunks():
    T, E, K = 20011, 200, 3
    x = torch.randn(T, E, generator=_gen(12), device="cuda")
    x[:, 50:] -= 100.0                                   # most experts get nothing
    ids, w, offsets, rows, source = pkg.asgd_route(x, K, align=128)
    flat = ids.reshape(-1).long()
    n = torch.bincount(flat, minlength=E)
    pad = (n + 127) // 128 * 128
    assert torch.equal(offsets.long(), torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), pad.cumsum(0)]))
    order = torch.sort(flat, stable=True).indices
    first = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), n.cumsum(0)])
    place = offsets[flat[order]].long() + torch.arange(T * K, device="cuda") - first[flat[order]]
    assert torch.equal(rows.reshape(-1)[order].long(), place)
    want = torch.full((source.numel(),), -1, dtype=torch.long, device="cuda")
    want[place] = order
    assert torch.equal(source.long(), want)


@pytest.mark.parametrize("T, E, K", [(41273, 70, 2), (41273, 24, 2), (18969, 300, 1)])
def test_route_plan_over_more_blocks_than_run_at_once(T, E, K):
    x = torch.rand(T, E, generator=_gen(T + E), device="cuda").argsort(dim=1).float()          # a permutation a row: no ties
    ids, w, offsets, rows, source = pkg.asgd_route(x, K, align=8)
    assert torch.equal(ids.long(), torch.topk(x, K).indices)
    flat = ids.reshape(-1).long()
    pad = (torch.bincount(flat, minlength=E) + 7) // 8 * 8
    assert torch.equal(offsets.long(), torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), pad.cumsum(0)]))
    order = torch.sort(flat, stable=True).indices
    want = torch.full((source.numel(),), -1, dtype=torch.long, device="cuda")
    first = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.bincount(flat, minlength=E).cumsum(0)])
    want[offsets[flat[order]].long() + torch.arange(T * K, device="cuda") - first[flat[order]]] = order
    assert torch.equal(source.long(), want)
    assert torch.equal(source.long()[rows.reshape(-1).long()], torch.arange(T * K, device="cuda"))


@pytest.mark.parametrize("T, E, top_k, score, dtype, renormalise", [
    (1, 4, 2, "softmax", F32, True), (67, 60, 6, "sigmoid", F32, True), (33, 129, 8, "softmax", BF, True), (33, 129, 8, "softmax", F32, False),
    (20, 256, 1, "sigmoid", F16, False), (9, 1000, 32, "softmax", F32, True), (12, 32, 32, "softmax", F32, True)])
def test_route_grad(T, E, top_k, score, dtype, renormalise):
    g = _gen(E + T)
    big = (torch.randn(T, E + 3, generator=g, device="cuda") * 2).to(dtype)
    x = big[:, 1:E + 1]
    ids, _ = pkg.asgd_route(x, top_k, score=score, plan=False)
    if T > 5:
        ids[3, top_k - 1] = -1                           # a place that was dropped
        ids[4] = -1
    dw = torch.randn(T, top_k, generator=g, device="cuda")
    got = pkg.asgd_route_grad(x, ids, dw, score=score, renormalise=renormalise, scale=1.7)
    z = x.double().requires_grad_()
    p = 1 / (1 + torch.exp(-z)) if score == "sigmoid" else torch.softmax(z, 1)
    c = p.gather(1, ids.long().clamp_min(0)) * (ids >= 0)
    w = 1.7 * c / (c.sum(1, keepdim=True) + 1e-20) if renormalise else 1.7 * c
    (want,) = torch.autograd.grad((w * dw.double()).sum(), z)
    # every term of the gradient is a product of scores (SCORE_TOL each, a few of them) and |dw| <= max; terms cancel
    most = 1.7 * dw.double().abs().amax(1, keepdim=True)
    bound = 8 * SCORE_TOL * (top_k + 2) * most * (p.detach() if score == "softmax" else 1.0) + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype] + 1e-12
    if renormalise and score == "sigmoid":
        total = c.detach().sum(1, keepdim=True)
        bound = bound / torch.clamp(total, max=1.0).clamp_min(1e-3)
    elif renormalise:
        bound = bound / c.detach().sum(1, keepdim=True).clamp_min(1e-6)
    assert got.dtype == dtype
    _close(got, want, bound)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_grad_against_differences(score):
    # well separated logits, so that a step changes no choice; h^2 / 6 of the third derivative (at most 1 of a weight
    # of size 1) and 2 * SCORE_TOL / (2 h) of rounding: below 2e-5 + 2e-3 with h = 2^-6... the sum over top_k weights
    T, E, K, h = 4, 12, 3, 2.0 ** -6
    g = _gen(21)
    x = (torch.rand(T, E, generator=g, device="cuda").argsort(1).float() - 6) * 0.25
    dw = torch.randn(T, K, generator=g, device="cuda")
    ids, _ = pkg.asgd_route(x, K, score=score, plan=False)
    got = pkg.asgd_route_grad(x, ids, dw, score=score)

    def value(v):
        i, w = pkg.asgd_route(v, K, score=score, plan=False)
        assert torch.equal(i, ids)
        return (w.double() * dw.double()).sum(1)
    for e in range(E):
        step = torch.zeros_like(x)
        step[:, e] = h
        diff = (value(x + step) - value(x - step)) / (2 * h)
        _close(got[:, e], diff, (h * h + 2 * SCORE_TOL / h) * dw.double().abs().sum(1))


# ---------------------------------------------------------------------------------------------------------------
# 8-bit operands
# ---------------------------------------------------------------------------------------------------------------

def _check_rounded(x, q, scale, bm, bn):
    """q * scale is x rounded, and the scale is the block's largest magnitude over the type's (x in fp64)."""
    M, K = x.shape
    F = FMAX[q.dtype]
    pad = torch.nn.functional.pad(x.abs(), (0, -K % bn, 0, -M % bm))
    amax = pad.reshape(pad.shape[0] // bm, bm, pad.shape[1] // bn, bn).amax(dim=(1, 3)).clamp_min(2.0 ** -100)
    assert scale.shape == amax.shape and q.shape == x.shape
    _close(scale, amax / F, 2 * U * amax / F)                          # 1 / F and the product are rounded
    s = scale.double().repeat_interleave(bm, 0)[:M].repeat_interleave(bn, 1)[:, :K]
    # half a step of the type at the quotient, or half its smallest step; F / a, the product and the scale are rounded (4 u)
    smallest = 2.0 ** -10 if q.dtype == E4 else 2.0 ** -17
    _close(q.float().double() * s, x, HALF_STEP[q.dtype] * x.abs() * (1 + 2 ** -3) + smallest * s * (1 + 8 * U) + 8 * U * x.abs())
    # not a step more than rounding to nearest takes: over many numbers the mean squared error is that of the type
    if x.numel() >= 10000:
        want = (x / s).float().to(q.dtype).float().double() * s
        err = lambda v: float(((v - x) ** 2).sum())                    # noqa: E731
        assert err(q.float().double() * s) <= err(want) * (1 + 1e-3)


def _numbers(M, K, dtype, seed):
    g = _gen(seed)
    x = torch.randn(M, K, generator=g, device="cuda") * torch.exp(2 * torch.randn(M, 1, generator=g, device="cuda"))
    x[:, ::13] *= 20
    if M > 2:
        x[1] = 0.0
        x[2, : K // 2] *= 1e-3
    return x.to(dtype)


@pytest.mark.parametrize("M, K, dtype, fmt", [(1, 1, F32, E4), (1, 128, BF, E4), (3, 129, F16, E5), (7, 1000, BF, E4), (130, 513, F32, E5),
                                              (129, 2048, BF, E5), (257, 136, F16, E4), (64, 4099, F32, E4)])
def test_quantize(M, K, dtype, fmt):
    x = _numbers(M, K, dtype, M + K)
    x64 = x.double()
    q, s = pkg.asgd_quantize(x, dtype=fmt)
    _check_rounded(x64, q, s, 1, 128)
    q2, s2, qt, st = pkg.asgd_quantize(x, form="both", dtype=fmt)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, s)
    _check_rounded(x64.t(), qt, st, 1, 128)
    qt3, st3 = pkg.asgd_quantize(x, form="columns", dtype=fmt)
    assert torch.equal(qt3.view(torch.uint8), qt.view(torch.uint8)) and torch.equal(st3, st)
    qb, sb = pkg.asgd_quantize(x, form="blocks", dtype=fmt)
    _check_rounded(x64, qb, sb, 128, 128)
    qb2, sb2, qbt = pkg.asgd_quantize(x, form="blocks both", dtype=fmt)
    assert torch.equal(qb2.view(torch.uint8), qb.view(torch.uint8)) and torch.equal(sb2, sb)
    assert torch.equal(qbt.view(torch.uint8), qb.view(torch.uint8).t())


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("K", [128, 200, 777])
def test_quantize_gathers_and_weighs(dtype, K):
    T, per = 50, 3
    x = _numbers(T, K, dtype, K)
    g = _gen(3)
    source = torch.randperm(T * per, generator=g, device="cuda").to(torch.int32)
    source = torch.cat([source[:60], torch.full((30,), -1, dtype=torch.int32, device="cuda"), source[60:],
                        torch.tensor([T * per, 2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")])      # beyond the input: zeros
    w = torch.randn(T, per, generator=g, device="cuda")
    there = (source >= 0) & (source < T * per)
    src = torch.where(there, source, torch.zeros_like(source)).long()
    for weights in (None, w):
        want = x.double()[src // per]
        if weights is not None:
            want = (x.float()[src // per] * w.reshape(-1)[src][:, None]).double()       # the product is rounded to fp32
        want = want * there[:, None]
        q, s, qt, st = pkg.asgd_quantize(x, form="both", source=source, per_token=per, weights=weights)
        _check_rounded(want, q, s, 1, 128)
        _check_rounded(want.t(), qt, st, 1, 128)
        q1, s1 = pkg.asgd_quantize(x, source=source, per_token=per, weights=weights)
        assert torch.equal(q1.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s1, s)


def test_quantize_strides_and_order():
    big = _numbers(70, 1003, BF, 4)
    for x in (big[:, 5:901], big[::2, 8:520], big[3:4, :], big.t().contiguous().t()[:, :1]):
        want = pkg.asgd_quantize(x.contiguous(), form="both")
        got = pkg.asgd_quantize(x, form="both")
        assert all(torch.equal(a.view(torch.uint8) if a.element_size() == 1 else a, b.view(torch.uint8) if b.element_size() == 1 else b)
                   for a, b in zip(got, want))
    with pytest.raises(ValueError):
        pkg.asgd_quantize(big.t())


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("K", [1, 7, 130, 1031])
def test_quantize_rows_that_start_anywhere(K, dtype):
    M, per = 37, 2
    big = _numbers(1, 8 + M * K, dtype, K)[0]
    source = torch.randperm(M * per, generator=_gen(K), device="cuda").to(torch.int32)
    wide = torch.zeros(M, -(-K // 16) * 16, dtype=dtype, device="cuda")
    for first in (0, 1, 2, 3, 5, 8):
        x = big[first:first + M * K].view(M, K)          # up to the storage's very end with first = 8
        wide[:, :K] = x
        for kw in (dict(form="both"), dict(form="blocks both"), dict(source=source, per_token=per), dict(form="both", source=source, per_token=per)):
            for got, want in zip(pkg.asgd_quantize(x, **kw), pkg.asgd_quantize(wide[:, :K], **kw)):
                one = got.element_size() == 1
                assert torch.equal(got.view(torch.uint8) if one else got, want.view(torch.uint8) if one else want)


def test_quantize_infinity_nan_and_tiny():
    x = torch.ones(4, 256, device="cuda")
    x[0, 3] = math.inf
    x[1, 200] = math.nan
    x[2] = 1e-35
    q, s = pkg.asgd_quantize(x)
    f = q.float()
    assert math.isinf(float(s[0, 0])) and torch.isnan(f[0, 3]) and (f[0, 4:128] == 0).all() and (f[0, 128:] == 448).all()
    assert torch.isnan(f[1, 200]) and (f[1, 128:200] == 448).all()
    assert torch.isfinite(s[1:]).all()
    # scaled by 2^-100: 1e-35 is 0.0057 of a step of 1, within half the type's smallest step (2^-9)
    _close(f[2, :128].double() * s[2, 0].double(), x[2, :128].double(), 2.0 ** -10 * s[2, 0].double() * (1 + 8 * U))
    assert pkg.asgd_quantize(x[:0])[0].shape == (0, 256)


# ---------------------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------------------

def _operand(rows, K, fmt, seed, square=False, lead=()):
    g = _gen(seed)
    kb = -(-K // 128)
    x = torch.randn(*lead, rows, K, generator=g, device="cuda") * FMAX[fmt] / 8
    q = torch.zeros(*lead, rows, -(-K // 16) * 16, dtype=torch.uint8, device="cuda")
    q[..., :K] = x.clamp(-FMAX[fmt], FMAX[fmt]).to(fmt).view(torch.uint8)
    s = torch.exp(torch.randn(*lead, -(-rows // 128) if square else rows, kb, generator=g, device="cuda")) / FMAX[fmt]
    return q[..., :K].view(fmt), s


def _values64(q, s):
    rows, K = q.shape[-2:]
    s = s.double()
    if s.shape[-2] != rows:
        s = s.repeat_interleave(128, -2)[..., :rows, :]
    return q.float().double() * s.repeat_interleave(128, -1)[..., :K]


def _check_product(c, a64, b64, K, dtype):
    want = a64 @ b64.t()
    # 128 products and additions of a block (any order, the tensor core's sums taken as fp32 ones), then two products
    # and an addition a block
    n = min(K, 128) + 4 * (-(-K // 128)) + 4
    bound = n * U * (a64.abs() @ b64.abs().t()) * 1.01
    _close(c, want, bound + HALF_STEP[dtype] * (want.abs() + bound) + SMALLEST[dtype])


@pytest.mark.parametrize("M, N, K, fa, fb, out, square", [
    (1, 1, 1, E4, E4, F32, False), (1, 128, 128, E4, E4, BF, True), (5, 200, 400, E4, E4, F32, True), (16, 130, 144, E5, E4, F16, True),
    (17, 256, 1040, E4, E5, F32, True), (33, 64, 2000, E5, E5, F32, False), (64, 257, 640, E4, E4, BF, False), (65, 384, 512, E4, E4, F32, True),
    (129, 513, 1000, E4, E4, F32, True), (300, 1000, 272, E5, E4, F32, False), (1000, 136, 777, E4, E4, BF, True), (513, 1100, 1536, E4, E4, F32, True),
    (257, 2048, 4096, E4, E5, F16, True), (700, 640, 384, E4, E4, F32, False), (2500, 2100, 300, E4, E4, F32, True)])
def test_product(M, N, K, fa, fb, out, square):
    a, sa = _operand(M, K, fa, 1)
    b, sb = _operand(N, K, fb, 2, square)
    c = pkg.asgd_product(a, sa, b, sb, out_dtype=out)
    _check_product(c, _values64(a, sa), _values64(b, sb), K, out)
    assert torch.equal(c, pkg.asgd_product(a, sa, b, sb, out_dtype=out))          # no sum depends on timing
    pkg.asgd_experts_sync()


def test_product_without_inner_dimension_or_rows():
    z = torch.zeros(5, 0, dtype=torch.uint8, device="cuda").view(E4)
    s = torch.zeros(5, 0, device="cuda")
    c = pkg.asgd_product(z, s, z, s, out=torch.full((5, 5), 7.0, device="cuda"))
    assert (c == 0).all()
    a, sa = _operand(4, 256, E4, 1)
    assert pkg.asgd_product(a[:0], sa[:0], a, sa).shape == (0, 4)


def test_product_strides():
    a, sa = _operand(150, 512, E4, 1)
    b, sb = _operand(300, 512, E4, 2, True)
    want = pkg.asgd_product(a, sa, b, sb, out_dtype=F32)
    big = torch.zeros(300, 800, dtype=torch.uint8, device="cuda").view(E4)
    big[::2, 16:528] = a
    scales = torch.zeros(8, 301, device="cuda")
    scales[::2, 1:151] = sa.t()
    out = torch.full((150, 333), -1.0, device="cuda")
    got = pkg.asgd_product(big[::2, 16:528], scales[::2, 1:151].t(), b, sb.t().contiguous().t(), out=out[:, 1:301])
    assert torch.equal(got, want) and (out[:, 0] == -1).all() and (out[:, 301:] == -1).all()
    with pytest.raises(binding.AsgdError):
        pkg.asgd_product(big[::2, 8:520], sa, b, sb)                              # not a 16-byte boundary
    with pytest.raises(ValueError):
        pkg.asgd_product(a, sa[:, :3], b, sb)


def test_product_propagates_nan_and_infinite_scales():
    a, sa = _operand(40, 256, E4, 1)
    b, sb = _operand(130, 256, E4, 2, True)
    sa[3, 1] = math.inf
    a.view(torch.uint8)[7, 9] = 0x7F                                              # NaN
    c = pkg.asgd_product(a, sa, b, sb, out_dtype=F32)
    keep = [r for r in range(40) if r not in (3, 7)]
    assert torch.isnan(c[7]).all() and not torch.isfinite(c[3]).any() and torch.isfinite(c[keep]).all()


def _loads(G, rows, seed, unit=1):
    """Rows per group: none, one, a few and many."""
    g = torch.Generator().manual_seed(seed)
    p = torch.rand(G, generator=g) ** 3
    if G > 1:
        p[G // 2] = 0.0
    n = torch.bincount(torch.multinomial(p, rows // unit, replacement=True, generator=g), minlength=G) * unit
    return torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)])


@pytest.mark.parametrize("G, M, N, K, out, square", [
    (1, 40, 128, 256, F32, True), (8, 8, 200, 384, F32, True), (8, 100, 200, 400, F32, True), (16, 700, 264, 640, BF, True), (5, 900, 136, 272, F32, False),
    (64, 500, 256, 128, F16, True), (8, 3000, 520, 512, F32, True), (300, 1000, 128, 144, F32, True), (4, 2600, 1100, 1040, F32, True)])
def test_product_grouped_over_rows(G, M, N, K, out, square):
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, square, (G,))
    at = _loads(G, M, G + M)
    at = torch.minimum(at, torch.tensor(M - M // 8))                               # the last rows are of no group
    c = torch.full((M, N), 3.0, dtype=out, device="cuda")
    pkg.asgd_product(a, sa, b, sb, offsets=at.to(torch.int32).cuda(), out=c)
    a64, b64, at = _values64(a, sa), _values64(b, sb), at.tolist()
    for g in range(G):
        if at[g + 1] > at[g]:
            _check_product(c[at[g]:at[g + 1]], a64[at[g]:at[g + 1]], b64[g], K, out)
    assert (c[at[G]:] == 3).all()
    pkg.asgd_experts_sync()


def test_product_grouped_with_strides_between_the_groups():
    G, M, N, K = 3, 90, 144, 256
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, True, (2 * G,))
    off = torch.tensor([0, 30, 30, 90], dtype=torch.int32, device="cuda")
    got = pkg.asgd_product(a, sa, b[1::2], sb[1::2], offsets=off)
    assert torch.equal(got, pkg.asgd_product(a, sa, b[1::2].contiguous(), sb[1::2].contiguous(), offsets=off))


@pytest.mark.parametrize("G, R, M, N, out, fa", [
    (1, 128, 128, 128, F32, E4), (4, 1024, 200, 136, F32, E5), (8, 640, 65, 300, BF, E4), (2, 4096, 513, 264, F32, E4), (16, 2048, 1, 1, F32, E4),
    (3, 1280, 600, 1000, F32, E5)])
def test_product_grouped_over_the_inner_dimension(G, R, M, N, out, fa):
    a, sa = _operand(M, R, fa, 1)
    b, sb = _operand(N, R, E4, 2)
    at = _loads(G, R, G + R, 128)
    c = pkg.asgd_product_inner(a, sa, b, sb, at.to(torch.int32).cuda(), out_dtype=out)
    a64, b64, at = _values64(a, sa), _values64(b, sb), at.tolist()
    for g in range(G):
        s = slice(at[g], at[g + 1])
        _check_product(c[g], a64[:, s], b64[:, s], at[g + 1] - at[g], out)
    pkg.asgd_experts_sync()


def test_inner_groups_may_end_at_the_matrix_and_nowhere_else():
    a, sa = _operand(70, 400, E4, 1)
    b, sb = _operand(90, 400, E4, 2)
    c = pkg.asgd_product_inner(a, sa, b, sb, torch.tensor([0, 128, 400], dtype=torch.int32, device="cuda"))
    a64, b64 = _values64(a, sa), _values64(b, sb)
    _check_product(c[0], a64[:, :128], b64[:, :128], 128, F32)
    _check_product(c[1], a64[:, 128:], b64[:, 128:], 272, F32)
    pkg.asgd_experts_sync()
    c = pkg.asgd_product_inner(a, sa, b, sb, torch.tensor([0, 100, 400], dtype=torch.int32, device="cuda"))
    assert torch.isnan(c).all()
    with pytest.raises(binding.AsgdError) as err:
        pkg.asgd_experts_sync()
    assert err.value.status == binding.ASGD_EINVAL
    pkg.asgd_experts_sync()                                                        # reported once


def test_offsets_beyond_the_matrix_are_cut():
    a, sa = _operand(40, 128, E4, 1)
    b, sb = _operand(128, 128, E4, 2, True, (3,))
    c = torch.full((40, 128), 3.0, device="cuda")
    pkg.asgd_product(a, sa, b, sb, offsets=torch.tensor([-7, 10, 900, 1000], dtype=torch.int32, device="cuda"), out=c)
    a64, b64 = _values64(a, sa), _values64(b, sb)
    _check_product(c[:10], a64[:10], b64[0], 128, F32)
    _check_product(c[10:], a64[10:], b64[1], 128, F32)


@pytest.mark.parametrize("M, N", [(8, 512), (60, 512), (600, 1024), (5000, 2048)])
def test_a_wait_that_runs_out_is_reported_and_the_device_stays_usable(M, N):
    a, sa = _operand(M, 1024, E4, 1)
    b, sb = _operand(N, 1024, E4, 2, True)
    want = pkg.asgd_product(a, sa, b, sb)
    pkg.asgd_experts_sync()
    try:
        pkg.asgd_product_set_wait_drill(2000, True)
        pkg.asgd_product(a, sa, b, sb)
        with pytest.raises(binding.AsgdError) as err:
            pkg.asgd_experts_sync()
        assert err.value.status == binding.ASGD_ETIMEOUT
    finally:
        pkg.asgd_product_set_wait_drill()
    assert torch.equal(pkg.asgd_product(a, sa, b, sb), want)
    pkg.asgd_experts_sync()


# ---------------------------------------------------------------------------------------------------------------
# combination
# ---------------------------------------------------------------------------------------------------------------

def _combine_case(T, D, K, dtype, R, seed):
    g = _gen(seed)
    z = torch.randn(R, D, generator=g, device="cuda").to(dtype)
    rows = torch.randperm(R, generator=g, device="cuda")[:T * K].reshape(T, K).to(torch.int32)
    w = torch.randn(T, K, generator=g, device="cuda")
    dy = torch.randn(T, D, generator=g, device="cuda").to(dtype)
    if T > 4:
        rows[2] = -1                                     # a token with no row
        rows[3, K - 1] = -1
        rows[4, 0] = R                                   # beyond z: no part
    return z, rows, w, dy


@pytest.mark.parametrize("T, D, K, dtype", [(1, 1, 1, F32), (1, 4096, 8, BF), (9, 130, 3, F16), (33, 1000, 4, F32), (70, 2056, 6, BF),
                                            (21, 515, 9, F16), (6, 264, 32, F32), (300, 64, 2, BF)])
def test_combine_and_gradient(T, D, K, dtype):
    R = T * K + 37
    z, rows, w, dy = _combine_case(T, D, K, dtype, R, T + D)
    there = (rows >= 0) & (rows < R)
    at = torch.where(there, rows, torch.zeros_like(rows)).long()
    source = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    source[at[there]] = torch.arange(T * K, dtype=torch.int32, device="cuda").reshape(T, K)[there]
    for weights in (w, None):
        f = (weights.double() if weights is not None else torch.ones(T, K, dtype=torch.float64, device="cuda")) * there
        zz = z.double()[at]
        want = (f[..., None] * zz).sum(1)
        bound = (K + 1) * U * (f[..., None] * zz).abs().sum(1)
        _close(pkg.asgd_combine(z, rows, weights), want, bound + HALF_STEP[dtype] * (want.abs() + bound) + SMALLEST[dtype])
        dz, dw = pkg.asgd_combine_grad(dy, z, rows, weights, source)
        terms = dy.double()[:, None] * zz * there[..., None]
        _close(dw, terms.sum(2), (D + 1) * U * terms.abs().sum(2))
        want = torch.zeros(R, D, dtype=torch.float64, device="cuda")
        want[at[there]] = (f[..., None] * dy.double()[:, None])[there]
        _close(dz, want, (HALF_STEP[dtype] + 2 * U) * want.abs() + SMALLEST[dtype])
    only = pkg.asgd_combine_grad(dy, z, rows, w, source, need_dz=False)
    assert only[0] is None and torch.equal(only[1], pkg.asgd_combine_grad(dy, z, rows, w, source)[1])
    assert pkg.asgd_combine_grad(dy, z, rows, w, source, need_dweights=False)[1] is None


def test_combine_strides_and_empty():
    z, rows, w, dy = _combine_case(40, 256, 3, BF, 130, 1)
    big = torch.zeros(130, 300, dtype=BF, device="cuda")
    for first in (8, 3):                                 # with and without whole 16-byte pieces
        big[:, first:first + 256] = z
        assert torch.equal(pkg.asgd_combine(big[:, first:first + 256], rows, w), pkg.asgd_combine(z, rows, w))
        got, want = pkg.asgd_combine_grad(dy, big[:, first:first + 256], rows, w, torch.full((130,), -1, dtype=torch.int32, device="cuda")), None
        want = pkg.asgd_combine_grad(dy, z, rows, w, torch.full((130,), -1, dtype=torch.int32, device="cuda"))
        _close(got[1], want[1], 2 * 257 * U * want[1].double().abs().max() * 40)
    assert pkg.asgd_combine(z, rows[:0]).shape == (0, 256)
    assert (pkg.asgd_combine(z[:0], rows, w) == 0).all()


def test_combine_gradient_against_differences():
    # y is linear in z and in the weights: a difference quotient is exact but for the rounding of y (fp32, u * |y| a term)
    T, D, K, R = 6, 40, 3, 20
    z, rows, w, dy = _combine_case(T, D, K, F32, R, 2)
    dz, dw = pkg.asgd_combine_grad(dy, z, rows, w, torch.zeros(R, dtype=torch.int32, device="cuda"))
    value = lambda zz, ww: (pkg.asgd_combine(zz, rows, ww).double() * dy.double()).sum()           # noqa: E731
    size = float((pkg.asgd_combine(z.abs(), rows, w.abs()).double() * dy.double().abs()).sum())
    h, tol = 0.5, 8 * U * size / 0.5 * 4
    for r in rows.flatten().tolist()[:6]:
        if not 0 <= r < R:
            continue
        step = torch.zeros_like(z)
        step[r, 7] = h
        assert abs(float(value(z + step, w) - value(z - step, w)) / (2 * h) - float(dz[r, 7])) <= tol
    for t, j in ((0, 0), (1, 2), (3, 1)):
        step = torch.zeros_like(w)
        step[t, j] = h
        assert abs(float(value(z, w + step) - value(z, w - step)) / (2 * h) - float(dw[t, j])) <= tol


# ---------------------------------------------------------------------------------------------------------------
# sizes beyond 32 bits, streams, and the whole path
# ---------------------------------------------------------------------------------------------------------------

def test_rows_beyond_two_to_the_31_numbers():
    R, D = 530_000, 4096                                 # 2.17e9 numbers
    z = torch.zeros(R, D, dtype=BF, device="cuda")
    z[-3:] = torch.randn(3, D, device="cuda").to(BF)
    rows = torch.tensor([[R - 1, 0], [R - 3, R - 2]], dtype=torch.int32, device="cuda")
    y = pkg.asgd_combine(z, rows)
    assert torch.equal(y[0], z[R - 1]) and torch.equal(y[1], (z[R - 3].float() + z[R - 2].float()).to(BF))
    q, s = pkg.asgd_quantize(z)
    _check_rounded(z[-3:].double(), q[-3:], s[-3:], 1, 128)
    source = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    source[[R - 1, 0, R - 3, R - 2]] = torch.arange(4, dtype=torch.int32, device="cuda")
    dy = torch.randn(2, D, device="cuda").to(BF)
    dz, dw = pkg.asgd_combine_grad(dy, z, rows, None, source)
    assert torch.equal(dz[R - 1], dy[0]) and torch.equal(dz[R - 3], dy[1])
    del dz
    b, sb = _operand(130, D, E4, 2, True)
    c = pkg.asgd_product(q, s, b, sb, out_dtype=F32)
    _check_product(c[-3:], _values64(q[-3:], s[-3:]), _values64(b, sb), D, F32)
    pkg.asgd_experts_sync()


def test_other_streams():
    a, sa = _operand(200, 512, E4, 1)
    b, sb = _operand(256, 512, E4, 2, True)
    z, rows, w, dy = _combine_case(40, 256, 3, BF, 130, 1)
    side = torch.cuda.Stream()
    want = (pkg.asgd_product(a, sa, b, sb), pkg.asgd_combine(z, rows, w), pkg.asgd_quantize(z)[1])
    side.wait_stream(torch.cuda.current_stream())
    got = (pkg.asgd_product(a, sa, b, sb, stream=side), pkg.asgd_combine(z, rows, w, stream=side), pkg.asgd_quantize(z, stream=side)[1])
    pkg.asgd_experts_sync(stream=side)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_can_be_captured_in_a_graph():
    x = torch.randn(90, 64, device="cuda")
    a, sa = _operand(180, 512, E4, 1)
    b, sb = _operand(128, 512, E4, 2, True, (64,))

    def step():
        ids, w, offsets, rows, source = pkg.asgd_route(x, 2)
        c = pkg.asgd_product(a, sa, b, sb, offsets=offsets)
        return pkg.asgd_combine(c, rows, w)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    x.copy_(torch.randn(90, 64, device="cuda"))
    g.replay()
    assert torch.equal(got, step())
