"""The operators of a layer of experts where tiles, groups and storage meet awkwardly, against 64 bits.  Bounds are those of
test_gpu_experts.py."""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding

from .test_gpu_experts import (BF, E4, E5, F16, F32, HALF_STEP, SCORE_TOL, SMALLEST, U, _check_product, _check_rounded, _close, _combine_case,
                               _gen, _loads, _numbers, _operand, _route_check, _values64)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------
# products: pairs of blocks that take several tiles in turn (74 pairs)
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G, R, M, N, out, fa", [
    (48, 48 * 128, 600, 520, F32, E4), (48, 48 * 128, 600, 520, BF, E5), (40, 40 * 128, 344, 1032, F16, E4), (64, 64 * 128, 600, 776, F32, E5)])
def test_inner_groups_without_rows_between_full_ones(G, R, M, N, out, fa):
    # 400 to 770 pair tiles; the last tile row is ragged, so that a warp writes C itself right after copies of a whole tile,
    # and a group of nothing has no K block between the two
    a, sa = _operand(M, R, fa, 1)
    b, sb = _operand(N, R, E4, 2)
    at = _loads(G, R, G + M, 128)
    empty = sum(int(p == q) for p, q in zip(at.tolist(), at.tolist()[1:]))
    assert empty >= G // 4
    a64, b64 = _values64(a, sa), _values64(b, sb)
    offsets, at = at.to(torch.int32).cuda(), at.tolist()
    first = None
    for _ in range(4):
        c = torch.full((G, M, N), 7.0, dtype=out, device="cuda")
        pkg.asgd_product_inner(a, sa, b, sb, offsets, out=c)
        if first is None:
            first = c
            for g in range(G):
                s = slice(at[g], at[g + 1])
                _check_product(c[g], a64[:, s], b64[:, s], at[g + 1] - at[g], out)
        assert torch.equal(c, first)
    pkg.asgd_experts_sync()


# ---------------------------------------------------------------------------------------------------------------
# products: scales and groups that start anywhere
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M, N, K, G", [(37, 136, 512, 3), (203, 264, 512, 4), (1900, 520, 256, 3), (2700, 1100, 1024, 3)])
@pytest.mark.parametrize("first", [0, 1, 2, 3])
def test_scales_and_groups_that_start_anywhere(M, N, K, G, first):
    # the scales lie `first` numbers behind a 16-byte boundary, block after block a whole number of 16 bytes apart, and the
    # groups start at rows of every remainder by 4: a tile's scales are aligned where the array of them is not
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, True, (G,))
    store = torch.zeros(K // 128 * 4096 + 8, device="cuda")
    moved = store[first:first + K // 128 * 4096].view(K // 128, 4096)[:, :M].t()
    moved.copy_(sa)
    assert moved.data_ptr() % 16 == 4 * first
    for start in range(4):
        at = torch.linspace(start, M, G + 1).to(torch.int32)
        at[1:-1] = at[1:-1] // 4 * 4 + (4 - first) % 4
        offsets = at.cuda()
        got = pkg.asgd_product(a, moved, b, sb, offsets=offsets, out=torch.zeros(M, N, device="cuda"))
        want = pkg.asgd_product(a, sa, b, sb, offsets=offsets, out=torch.zeros(M, N, device="cuda"))
        assert torch.equal(got, want)
        a64, b64, rows = _values64(a, sa), _values64(b, sb), at.tolist()
        for g in range(G):
            s = slice(rows[g], rows[g + 1])
            _check_product(got[s], a64[s], b64[g], K, F32)
    pkg.asgd_experts_sync()


# ---------------------------------------------------------------------------------------------------------------
# products: the most rows and columns
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("by_groups", [False, True])
def test_products_of_the_most_rows_and_columns(by_groups):
    n = 2 ** 31 - 256                                    # 34 GB of rows of 16 numbers
    long = torch.zeros(n, 16, dtype=torch.uint8, device="cuda")
    scale = torch.ones(n, 1, device="cuda")
    a, sa = _operand(300, 16, E4, 1)
    long[-300:] = a.view(torch.uint8)
    scale[-300:] = sa
    b, sb = _operand(1, 16, E4, 2)
    a64, b64 = _values64(a, sa), _values64(b, sb)
    out = torch.full((n, 1), 5.0, device="cuda")
    if by_groups:
        offsets = torch.tensor([0, 7, 7, n], dtype=torch.int32, device="cuda")
        pkg.asgd_product(long.view(E4), scale, b.view(torch.uint8).expand(3, 1, 16).contiguous().view(E4), sb.expand(3, 1, 1), offsets=offsets, out=out)
    else:
        pkg.asgd_product(long.view(E4), scale, b, sb, out=out)
    pkg.asgd_experts_sync()
    _check_product(out[-300:], a64, b64, 16, F32)
    assert int(out[:-300].count_nonzero()) == 0
    if by_groups:
        return
    out.fill_(5.0)
    pkg.asgd_product(b, sb, long.view(E4), scale, out=out.view(1, n))
    pkg.asgd_experts_sync()
    _check_product(out.view(1, n)[:, -300:], b64, a64, 16, F32)
    assert int(out[:-300].count_nonzero()) == 0


# ---------------------------------------------------------------------------------------------------------------
# reports
# ---------------------------------------------------------------------------------------------------------------

def test_no_report_is_lost_while_another_is_taken():
    # a wait that runs out on one stream, while calls on another stream report offsets that cut a block and are taken one
    # after the other: whichever call takes it, the timeout (the worse status) is seen
    a, sa = _operand(8, 1024, E4, 1)
    b, sb = _operand(512, 1024, E4, 2, True)
    u, su = _operand(16, 400, E4, 3)
    cut = torch.tensor([0, 100, 400], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    pkg.asgd_product(a, sa, b, sb)
    pkg.asgd_product_inner(u, su, u, su, cut[::2].contiguous())
    torch.cuda.synchronize()
    try:
        pkg.asgd_experts_sync()
    except binding.AsgdError:
        pass

    def take(stream=None):
        try:
            pkg.asgd_experts_sync(stream)
            return binding.ASGD_OK
        except binding.AsgdError as err:
            return err.status
    for _ in range(40):
        try:
            pkg.asgd_product_set_wait_drill(2000, True)
            pkg.asgd_product(a, sa, b, sb, stream=side)
        finally:
            pkg.asgd_product_set_wait_drill()
        seen, turns = [], 0
        while not side.query():
            pkg.asgd_product_inner(u, su, u, su, cut)
            seen.append(take())
            turns += 1
            assert turns < 10 ** 6
        seen.append(take(side))
        assert binding.ASGD_ETIMEOUT in seen             # (each of the call's blocks reports: more than one may see it)
        assert all(s == binding.ASGD_EINVAL for s in seen[:-1] if s != binding.ASGD_ETIMEOUT)
    assert take() == binding.ASGD_OK


# ---------------------------------------------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("E, top_k", [(12, 12), (40, 8), (200, 16), (1000, 32)])
def test_sigmoid_gradient_of_large_logits(E, top_k, dtype):
    # dx = scale * dw * s * (1 - s), relative to itself: both sigmoids (exponential 4 u, sum and reciprocal 1 u each), three
    # products and the factor scale * dw stay below 32 u
    g = _gen(E)
    T = 60
    size = 10 + 20 * torch.rand(T, E, generator=g, device="cuda")
    x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.5, size, -size).to(dtype)
    ids = torch.rand(T, E, generator=g, device="cuda").argsort(dim=1)[:, :top_k].to(torch.int32).contiguous()
    dw = torch.randn(T, top_k, generator=g, device="cuda")
    got = pkg.asgd_route_grad(x, ids, dw, score="sigmoid", renormalise=False, scale=1.5)
    z = x.double()
    want = torch.zeros_like(z).scatter(1, ids.long(), 1.5 * dw.double()) / ((1 + torch.exp(-z)) * (1 + torch.exp(z)))
    _close(got, want, (32 * U + HALF_STEP[dtype]) * want.abs() + SMALLEST[dtype])


@pytest.mark.parametrize("E, top_k, groups, kept", [(64, 12, 1, 1), (100, 8, 1, 1), (128, 8, 8, 3), (256, 10, 16, 4), (256, 32, 1, 1), (500, 6, 1, 1), (1024, 16, 32, 5)])
def test_ties_among_many_experts(E, top_k, groups, kept):
    # more equal keys than a warp has lanes, and rows with no more than a few experts
    x = torch.randint(0, 3, (150, E), generator=_gen(E + 1), device="cuda").float()
    x[0] = 1.0
    x[1] = -math.inf
    x[1, E // 2] = 0.0
    x[2, 3:] = -math.inf
    x[100:] = torch.where(torch.rand(50, E, generator=_gen(E + 2), device="cuda") < 0.9, torch.full((), -math.inf, device="cuda"), x[100:])
    _route_check(x, top_k, groups=groups, kept=kept, align=16, min_clear=1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T, E, top_k, dtype", [(70, 24, 3, F32), (45, 100, 8, F32), (45, 128, 4, BF), (30, 400, 10, F32), (30, 512, 2, F16), (35, 64, 9, F32)])
def test_route_grad_of_every_width(T, E, top_k, dtype, score):
    g = _gen(E)
    x = (torch.randn(T, E, generator=g, device="cuda") * 2).to(dtype)
    ids = torch.rand(T, E, generator=g, device="cuda").argsort(dim=1)[:, :top_k].to(torch.int32).contiguous()
    dw = torch.randn(T, top_k, generator=g, device="cuda")
    got = pkg.asgd_route_grad(x, ids, dw, score=score, renormalise=False, scale=1.7)
    z = x.double().requires_grad_()
    p = 1 / (1 + torch.exp(-z)) if score == "sigmoid" else torch.softmax(z, 1)
    (want,) = torch.autograd.grad((1.7 * p.gather(1, ids.long()) * dw.double()).sum(), z)
    most = 1.7 * dw.double().abs().amax(1, keepdim=True)
    bound = 8 * SCORE_TOL * (top_k + 2) * most * p.detach() + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype] + 1e-12
    _close(got, want, bound)


# ---------------------------------------------------------------------------------------------------------------
# the kernel instances of larger sizes
# ---------------------------------------------------------------------------------------------------------------

def _block_after_block(s):
    """Scales laid out as the quantiser leaves them: neighbouring rows' scales are neighbours in memory."""
    return s.transpose(-1, -2).contiguous().transpose(-1, -2)


@pytest.mark.parametrize("out", [F32, BF, F16])
@pytest.mark.parametrize("M, N, K, square", [(2305, 1040, 640, True), (2500, 1030, 300, True), (2311, 1544, 512, False), (2560, 2050, 144, False), (5003, 520, 400, True)])
def test_products_of_many_rows(M, N, K, square, out):
    # with rows of C at 16-byte boundaries and not; a scale per column and per 128 x 128; ragged last tiles both ways
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E5, 2, square)
    a64, b64 = _values64(a, sa), _values64(b, sb)
    c = pkg.asgd_product(a, sa, b, sb, out_dtype=out)
    _check_product(c, a64, b64, K, out)
    assert torch.equal(c, pkg.asgd_product(a, _block_after_block(sa), b, _block_after_block(sb), out_dtype=out))
    wide = torch.full((M, N + 41), 9.0, dtype=out, device="cuda")
    pkg.asgd_product(a, sa, b, sb, out=wide[:, 8:8 + N])
    assert torch.equal(wide[:, 8:8 + N], c) and bool((wide[:, :8] == 9).all()) and bool((wide[:, 8 + N:] == 9).all())
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("out", [F32, BF, F16])
@pytest.mark.parametrize("N, K, square", [(520, 512, True), (1100, 272, True), (776, 640, False)])
def test_groups_of_many_rows_that_end_anywhere(N, K, square, out):
    # 33 groups of 256 + r rows, r = 0..32, and one of nothing among them
    sizes = [256 + r for r in range(33)]
    sizes.insert(20, 0)
    at = torch.cat([torch.zeros(1, dtype=torch.long), torch.tensor(sizes).cumsum(0)])
    G, M = len(sizes), int(at[-1])
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, square, (G,))
    a64, b64 = _values64(a, sa), _values64(b, sb)
    offsets, at = at.to(torch.int32).cuda(), at.tolist()
    for scales in (sa, _block_after_block(sa)):
        c = pkg.asgd_product(a, scales, b, sb, offsets=offsets, out_dtype=out)
        for g in range(G):
            s = slice(at[g], at[g + 1])
            if at[g + 1] > at[g]:
                _check_product(c[s], a64[s], b64[g], K, out)
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("G, R, M, N, out, fa", [
    (6, 6144, 1112, 1032, F32, E4), (6, 6144, 1111, 1031, F32, E5), (5, 5000, 1290, 776, BF, E4), (5, 5000, 1290, 777, F16, E5), (16, 16384, 512, 1024, F32, E5)])
def test_inner_groups_of_many_columns(G, R, M, N, out, fa):
    a, sa = _operand(M, R, fa, 1)
    b, sb = _operand(N, R, E4, 2)
    at = _loads(G, R // 128 * 128, G + R, 128)
    at[-1] = R                                           # the last group may end inside a block of 128
    a64, b64 = _values64(a, sa), _values64(b, sb)
    offsets, at = at.to(torch.int32).cuda(), at.tolist()
    c = pkg.asgd_product_inner(a, sa, b, sb, offsets, out_dtype=out)
    for g in range(G):
        s = slice(at[g], at[g + 1])
        _check_product(c[g], a64[:, s], b64[:, s], at[g + 1] - at[g], out)
    assert torch.equal(c, pkg.asgd_product_inner(a, _block_after_block(sa), b, _block_after_block(sb), offsets, out_dtype=out))
    between = torch.full((M, G, N), 9.0, dtype=out, device="cuda").permute(1, 0, 2)                     # groups' rows in turn
    assert torch.equal(c, pkg.asgd_product_inner(a, sa, b, sb, offsets, out=between))
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("out", [F32, BF])
# tiles of 16, 32, 64 and 128 rows, a block each and shared by clusters of 2, 4 and 8
@pytest.mark.parametrize("M, N, K", [(600, 1024, 1024), (590, 1030, 1040), (250, 2056, 700), (678, 784, 1536), (594, 411, 1024), (529, 132, 2048),
                                     (5, 3, 512), (2, 18, 1024), (2, 6, 2048), (466, 514, 256), (660, 260, 1024), (582, 1, 1024), (345, 1, 2048),
                                     (514, 1027, 256), (261, 1286, 1536), (551, 129, 1024), (455, 1, 3200)])
def test_products_of_middling_rows(M, N, K, out):
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, True)
    c = pkg.asgd_product(a, sa, b, sb, out_dtype=out)
    _check_product(c, _values64(a, sa), _values64(b, sb), K, out)
    assert torch.equal(c, pkg.asgd_product(a, _block_after_block(sa), b, sb, out_dtype=out))
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("T, D, K, dtype", [(2500, 264, 2, BF), (1200, 130, 4, F32), (900, 1030, 6, F16), (5000, 512, 1, F32), (700, 2048, 8, BF)])
def test_combine_gradient_of_many_assignments(T, D, K, dtype):
    assert T * K >= 4736
    R = T * K + 261
    z, rows, w, dy = _combine_case(T, D, K, dtype, R, T + D)
    there = (rows >= 0) & (rows < R)
    at = torch.where(there, rows, torch.zeros_like(rows)).long()
    source = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    source[at[there]] = torch.arange(T * K, dtype=torch.int32, device="cuda").reshape(T, K)[there]
    dz, dw = pkg.asgd_combine_grad(dy, z, rows, w, source)
    terms = dy.double()[:, None] * z.double()[at] * there[..., None]
    _close(dw, terms.sum(2), (D + 1) * U * terms.abs().sum(2))
    del terms
    want = torch.zeros(R, D, dtype=torch.float64, device="cuda")
    want[at[there]] = ((w.double() * there)[..., None] * dy.double()[:, None])[there]
    _close(dz, want, (HALF_STEP[dtype] + 2 * U) * want.abs() + SMALLEST[dtype])
    only = pkg.asgd_combine_grad(dy, z, rows, w, source, need_dz=False)
    assert only[0] is None and torch.equal(only[1], dw)
    only = pkg.asgd_combine_grad(dy, z, rows, w, source, need_dweights=False)
    assert torch.equal(only[0], dz) and only[1] is None


@pytest.mark.parametrize("dtype, K", [(BF, 4096), (BF, 2048), (F16, 2056), (F32, 1024), (F32, 2600), (BF, 6008)])
@pytest.mark.parametrize("fmt", [E4, E5])
def test_quantize_gathers_many_long_rows(dtype, K, fmt):
    T, per = 230, 3
    x = _numbers(T, K, dtype, K)
    g = _gen(K + 1)
    source = torch.randperm(T * per, generator=g, device="cuda").to(torch.int32)
    source = torch.cat([source[:400], torch.full((57,), -1, dtype=torch.int32, device="cuda"), source[400:]])      # rows of nothing
    assert source.numel() >= 592
    w = torch.randn(T, per, generator=g, device="cuda")
    there, src = source >= 0, source.clamp_min(0).long()
    for weights in (None, w):
        want = x.double()[src // per]
        if weights is not None:
            want = (x.float()[src // per] * w.reshape(-1)[src][:, None]).double()
        q, s = pkg.asgd_quantize(x, dtype=fmt, source=source, per_token=per, weights=weights)
        _check_rounded(want * there[:, None], q, s, 1, 128)
        q2, s2, _, _ = pkg.asgd_quantize(x, form="both", dtype=fmt, source=source, per_token=per, weights=weights)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s, s2)


@pytest.mark.parametrize("T, E, top_k, D, N, popular", [(700, 20, 3, 272, 264, 6), (3000, 8, 2, 520, 400, 8), (40, 200, 4, 256, 136, 30)])
def test_a_padded_plan_is_fed_on(T, E, top_k, D, N, popular):
    # route with rows of 128 -> gathered both ways -> the experts' products and weight gradients -> back, and the gradient
    g = _gen(T + E)
    logits = torch.randn(T, E, generator=g, device="cuda")
    logits[:, popular:] -= 30.0                          # the other experts get nothing
    x = _numbers(T, D, BF, T)
    ids, w, offsets, rows, source = pkg.asgd_route(logits, top_k, align=128)
    R, at = source.numel(), offsets.tolist()
    there, src = source >= 0, source.clamp_min(0).long()
    assert bool((~there).any()) and at[E] < R
    xq, xs, xqt, xst = pkg.asgd_quantize(x, form="both", source=source, per_token=top_k)
    gathered = x.double()[src // top_k] * there[:, None]
    _check_rounded(gathered, xq, xs, 1, 128)
    _check_rounded(gathered.t(), xqt, xst, 1, 128)
    wq, ws = _operand(N, D, E4, 2, True, (E,))
    z = pkg.asgd_product(xq, xs, wq, ws, offsets=offsets, out_dtype=F32, out=torch.full((R, N), 4.0, device="cuda"))
    x64, w64 = _values64(xq, xs), _values64(wq, ws)
    for e in range(E):
        s = slice(at[e], at[e + 1])
        if at[e + 1] > at[e]:
            _check_product(z[s], x64[s], w64[e], D, F32)
    assert bool((z[at[E]:] == 4).all())
    assert not z[:at[E]][~there[:at[E]]].any()           # rows of nothing inside an expert
    at_rows = rows.long()
    f = w.double()[..., None] * z.double()[at_rows]
    y = pkg.asgd_combine(z, rows, w)
    _close(y, f.sum(1), (top_k + 2) * U * f.abs().sum(1))
    dy = torch.randn(T, N, generator=g, device="cuda")
    dz, dw = pkg.asgd_combine_grad(dy, z, rows, w, source)
    want = torch.zeros(R, N, dtype=torch.float64, device="cuda")
    want[at_rows] = w.double()[..., None] * dy.double()[:, None]
    _close(dz, want, 2 * U * want.abs())
    dzq, dzs, dzqt, dzst = pkg.asgd_quantize(dz, form="both", dtype=E5)
    _check_rounded(dz.double(), dzq, dzs, 1, 128)
    dwt = pkg.asgd_product_inner(dzqt, dzst, xqt, xst, offsets)
    a64, b64 = _values64(dzqt, dzst), _values64(xqt, xst)
    for e in range(E):
        s = slice(at[e], at[e + 1])
        _check_product(dwt[e], a64[:, s], b64[:, s], at[e + 1] - at[e], F32)
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("withhold", [False, True])
@pytest.mark.parametrize("M, N, K, inner", [(8, 512, 1024, 0), (5, 256, 512, 0), (60, 4096, 4096, 0), (600, 1024, 1024, 0), (2500, 2048, 2048, 0), (600, 520, 40 * 128, 40)])
def test_waits_given_up_at_any_time_leave_nothing_in_flight(M, N, K, inner, withhold):
    # a wait given up after a few polls runs out anywhere in the kernel, with copies and products on their way
    a, sa = _operand(M, K, E4, 1)
    b, sb = _operand(N, K, E4, 2, not inner)
    offsets = (torch.arange(inner + 1) * (K // max(inner, 1))).to(torch.int32).cuda()

    def call():
        if inner:
            return pkg.asgd_product_inner(a, sa, b, sb, offsets)
        return pkg.asgd_product(a, sa, b, sb, out_dtype=F32)
    want = call()
    pkg.asgd_experts_sync()
    ran_out = 0
    for limit in (1, 2, 3, 5, 9, 17, 40, 100, 300):
        try:
            pkg.asgd_product_set_wait_drill(limit, withhold)
            got = call()
            try:
                pkg.asgd_experts_sync()
                assert not withhold and torch.equal(got, want)
            except binding.AsgdError as err:
                assert err.status == binding.ASGD_ETIMEOUT
                ran_out += 1
        finally:
            pkg.asgd_product_set_wait_drill()
        assert torch.equal(call(), want)
        pkg.asgd_experts_sync()
    assert ran_out == 9 if withhold else ran_out <= 9
