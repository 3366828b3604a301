"""4-bit operands and products on the GPU against plain implementations in 64 bits.

Tolerances.  Rounding to 4 bits has none: the power of two and the rounding are defined exactly, and the kernel's scaling is exact.  In
a product the numbers' products are exact in fp32 (two bits by two bits, times powers of two); a sum of K of them in any order on the
tensor cores, each addition cut or rounded to fp32 (2 u, u = 2^-24), and the sums of eight blocks of a cluster (rounded) is within 2 (K + 8) u of the sum of the
magnitudes; C is then within half a step of its type of that.
"""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_STEP = {F32: U, BF: 2.0 ** -8, F16: 2.0 ** -11}
SMALLEST = {F32: 2.0 ** -149, BF: 2.0 ** -133, F16: 2.0 ** -24}
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _numbers(M, K, dtype, seed):
    g = _gen(seed)
    x = torch.randn(M, K, generator=g, device="cuda") * torch.exp(2 * torch.randn(M, 1, generator=g, device="cuda"))
    x[:, ::13] *= 16
    x[:, 5::29] = 0
    return x.to(dtype)


def _codes64(x):
    """Codes [M, K] (0 .. 15) and scale bytes [M, blocks] of x by the definition, block by block in 64 bits on the CPU."""
    x = x.double().cpu()
    M, K = x.shape
    codes, scale = torch.zeros(M, K, dtype=torch.int64), torch.zeros(M, -(-K // 32), dtype=torch.int64)
    for b in range(scale.shape[1]):
        v = x[:, 32 * b:32 * b + 32]
        bad = ~torch.isfinite(v).all(1)
        v = torch.where(bad[:, None], torch.zeros_like(v), v)
        a = v.abs().amax(1).clamp_min(2.0 ** -100)
        e = torch.full_like(a, -200.0)
        for k in range(-110, 130):                                     # the smallest power with a <= 6 * 2^k
            e = torch.where((e == -200.0) & (a <= 6 * 2.0 ** k), torch.full_like(e, float(k)), e)
        t = (v / torch.exp2(e)[:, None]).abs()
        far = torch.stack([(t - g).abs() for g in GRID], -1)
        best = far.amin(-1, keepdim=True)
        near = far == best                                             # two at a tie: the even one
        even = torch.tensor([0, 2, 4, 6])
        first = near.int().argmax(-1)
        tie_even = near[..., even].int().argmax(-1) * 2
        code = torch.where(near.sum(-1) == 2, tie_even, first)
        codes[:, 32 * b:32 * b + 32] = torch.where(bad[:, None], torch.zeros_like(code), code + 8 * torch.signbit(v).long())
        scale[:, b] = torch.where(bad, torch.full_like(a, 255.0), e + 127).long()
    return codes, scale


def _unpack(q, K):
    b = q.view(torch.uint8).cpu().long()
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)[..., :K]


def _check_rounded(x, q, scale):
    K = x.shape[1]
    codes, want = _codes64(x)
    assert torch.equal(scale.view(torch.uint8).cpu().long(), want)
    assert torch.equal(_unpack(q, K), codes)
    if K % 2:
        assert bool((q.view(torch.uint8)[:, -1] < 16).all())           # nothing behind an odd row


@pytest.mark.parametrize("M, K, dtype", [(1, 1, F32), (1, 32, BF), (3, 33, F16), (7, 1000, BF), (130, 513, F32), (129, 2048, BF), (257, 136, F16),
                                         (64, 1027, F32), (65, 1027, BF), (5, 8, F16), (9, 2, BF)])
def test_quantize4(M, K, dtype):
    x = _numbers(M, K, dtype, M + K)
    q, s = pkg.asgd_quantize4(x)
    assert q.shape == (M, -(-K // 2)) and s.shape == (M, -(-K // 32))
    _check_rounded(x, q, s)
    for out in (F32, BF, F16):
        got = pkg.asgd_dequantize4(q, s, K, dtype=out)
        v = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)[_unpack(q, K)]
        v = v * torch.exp2(s.view(torch.uint8).cpu().double() - 127).repeat_interleave(32, 1)[:, :K]
        assert got.shape == (M, K) and torch.equal(got.cpu().double(), v.float().to(out).double())       # fp32 holds them all


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize4_of_ties_and_borders(dtype):
    # the largest number at and beside 6, 3 and 8 steps, and every tie between two numbers of the grid, at several powers of two
    rows = []
    for top in (4.0, 5.9375, 6.0, 6.0625, 3.0, 3.03125, 3.5, 7.0, 7.9375, 1.0):
        for e in (-10, 0, 7):
            ties = [t * s for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.125, 0.5, 1.5) for s in (1, -1)]
            rows.append([top * 2.0 ** e] + [t * 2.0 ** e for t in ties if abs(t) <= top] + [0.0] * (31 - sum(abs(t) <= top for t in ties)))
    x = torch.tensor(rows, device="cuda").to(dtype)
    q, s = pkg.asgd_quantize4(x)
    _check_rounded(x, q, s)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("K", [32, 200, 777])
def test_quantize4_gathers_and_weighs(dtype, K):
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
        want = x.float()[src // per] * (1.0 if weights is None else w.reshape(-1)[src][:, None])          # the product is rounded to fp32
        want = torch.where(there[:, None], want, torch.zeros_like(want))
        q, s = pkg.asgd_quantize4(x, source=source, per_token=per, weights=weights)
        _check_rounded(want, q, s)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize4_strides_and_rows_that_start_anywhere(dtype):
    big = _numbers(70, 1003, dtype, 4)
    for x in (big[:, 5:901], big[::2, 8:520], big[3:4, :], big[:, 1:2], big[1:, :]):
        want = pkg.asgd_quantize4(x.contiguous())
        got = pkg.asgd_quantize4(x)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    flat = _numbers(1, 8 + 37 * 131, dtype, 9)[0]
    for first in (0, 1, 2, 3, 5, 8):
        x = flat[first:first + 37 * 131].view(37, 131)                 # up to the storage's very end with first = 8
        _check_rounded(x, *pkg.asgd_quantize4(x))
    with pytest.raises(ValueError):
        pkg.asgd_quantize4(big.t())


@pytest.mark.parametrize("K", [2, 6, 30, 130, 514, 1030, 4094])
def test_rows_of_32_bits_that_start_at_8_bytes(K):
    x = _numbers(37, K, F32, K)
    assert x.stride(0) % 4 == 2
    q, s = pkg.asgd_quantize4(x)
    wide_q, wide_s = pkg.asgd_quantize4(torch.nn.functional.pad(x, (0, 2)))
    assert torch.equal(q.view(torch.uint8), wide_q.view(torch.uint8)[:, :K // 2]) and torch.equal(s.view(torch.uint8), wide_s.view(torch.uint8)[:, :s.shape[1]])
    back = pkg.asgd_dequantize4(q, s, K, dtype=F32)
    assert torch.equal(back, pkg.asgd_dequantize4(wide_q, wide_s, K + 2, dtype=F32)[:, :K])
    shifted = torch.zeros(37 * K + 2, device="cuda")
    shifted[2:] = x.flatten()
    got = pkg.asgd_quantize4(shifted[2:].view(37, K))
    assert torch.equal(got[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got[1].view(torch.uint8), s.view(torch.uint8))


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize4_infinity_nan_and_extremes(dtype):
    x = torch.ones(6, 96, device="cuda", dtype=dtype)
    x[0, 3] = math.inf
    x[1, 40] = math.nan
    x[2, 95] = -math.inf
    x[3] = 0
    x[4] = torch.finfo(dtype).max
    x[5] = torch.finfo(dtype).tiny / 2                                 # scaled by 2^-100 at least
    q, s = pkg.asgd_quantize4(x)
    _check_rounded(x, q, s)
    v = pkg.asgd_dequantize4(q, s, dtype=F32)
    assert torch.isnan(v[0, :32]).all() and (v[0, 32:] == 1).all() and torch.isnan(v[1, 32:64]).all() and torch.isnan(v[2, 64:]).all()
    assert pkg.asgd_quantize4(x[:0])[0].shape == (0, 48)
    w = torch.full((6, 1), math.inf, device="cuda")
    q, s = pkg.asgd_quantize4(x, source=torch.arange(6, dtype=torch.int32, device="cuda"), weights=w)
    assert (s.view(torch.uint8) == 255).all() and (q.view(torch.uint8) == 0).all()                         # 0 * infinity among them


def test_dequantize4_strides_and_refusals():
    x = _numbers(40, 300, F32, 1)
    q, s = pkg.asgd_quantize4(x)
    want = pkg.asgd_dequantize4(q, s, 300)
    big = torch.full((40, 200), 255, dtype=torch.uint8, device="cuda")
    big[:, 3:153] = q.view(torch.uint8)
    scales = torch.full((40, 13), 255, dtype=torch.uint8, device="cuda")
    scales[:, 2:12] = s.view(torch.uint8)
    got = pkg.asgd_dequantize4(big[:, 3:153].view(q.dtype), scales[:, 2:12].view(s.dtype), 300)
    assert torch.equal(got, want)
    for bad in (301, 298, 0):
        with pytest.raises(ValueError):
            pkg.asgd_dequantize4(q, s, bad)
    with pytest.raises(ValueError):
        pkg.asgd_dequantize4(q, s[:, :9], 300)
    with pytest.raises(ValueError):
        pkg.asgd_dequantize4(q, s, 300, dtype=torch.float64)


# ---------------------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------------------

def _operand(rows, K, seed, lead=(), spread=3):
    """Any codes, and scales that differ from block to block."""
    g = _gen(seed)
    n, kb = -(-K // 2), -(-K // 32)
    q = torch.zeros(*lead, rows, -(-n // 16) * 16, dtype=torch.uint8, device="cuda")
    q[..., :n] = torch.randint(0, 256, (*lead, rows, n), generator=g, device="cuda", dtype=torch.uint8)
    if K % 2:
        q[..., n - 1] &= 15
    s = torch.full((*lead, rows, -(-kb // 16) * 16), 255, dtype=torch.uint8, device="cuda")              # NaN behind the last block
    s[..., :kb] = torch.randint(127 - spread, 128 + spread, (*lead, rows, kb), generator=g, device="cuda", dtype=torch.uint8)
    return q[..., :n].view(torch.float4_e2m1fn_x2), s[..., :kb].view(torch.float8_e8m0fnu)


def _values64(q, s):
    b = q.view(torch.uint8).long()
    v = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64, device="cuda")[torch.stack([b & 15, b >> 4], -1).flatten(-2)]
    return v * torch.exp2(s.view(torch.uint8).double() - 127).repeat_interleave(32, -1)[..., :v.shape[-1]]


def _check_product(c, a64, b64, dtype):
    want = a64 @ b64.t()
    bound = 2 * (a64.shape[1] + 8) * U * (a64.abs() @ b64.abs().t()) * 1.01
    assert c.dtype == dtype and not torch.isnan(c).any()
    off = (c.double() - want).abs() - (bound + HALF_STEP[dtype] * (want.abs() + bound) + SMALLEST[dtype])
    assert float(off.max()) <= 0.0, float(off.max())


# every kernel: few rows of 16, 32, 64 and 128 with and without a shared tile, and the pair; units of 512 numbers that end anywhere
SHAPES = [(1, 1, 1, F32), (1, 128, 32, BF), (5, 200, 400, F32), (16, 130, 144, F16), (17, 256, 1040, F32), (33, 64, 2000, F32), (64, 257, 640, BF),
          (65, 384, 512, F32), (129, 513, 1000, F32), (300, 1000, 272, F32), (1000, 136, 777, BF), (513, 1100, 1536, F32), (257, 2048, 4096, F16),
          (700, 640, 384, F32), (2500, 2100, 300, F32), (5, 4096, 4096, F32), (3, 96, 8192, F32), (1500, 4000, 64, F32), (1025, 2240, 2048, F32),
          (20, 4096, 1024, F32), (100, 4096, 2080, F32), (200, 4096, 4096, F32), (4096, 1024, 1090, BF)]


@pytest.mark.parametrize("M, N, K, out", SHAPES)
def test_product4(M, N, K, out):
    a, sa = _operand(M, K, 1)
    b, sb = _operand(N, K, 2)
    c = pkg.asgd_product4(a, sa, b, sb, out_dtype=out)
    pkg.asgd_experts_sync()
    _check_product(c, _values64(a, sa), _values64(b, sb), out)
    assert torch.equal(c, pkg.asgd_product4(a, sa, b, sb, out_dtype=out))          # no sum depends on timing
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("M, N", [(7, 130), (300, 2300)])
def test_every_scale_meets_its_own_numbers(M, N):
    # one number per row of A and one block per row of B: an entry of C shows one product of two scales
    K = 1088
    for k in list(range(0, K, 32)) + [31, 63, 500, 1087]:
        a = torch.zeros(M, K // 2, dtype=torch.uint8, device="cuda")
        a[:, k // 2] = 2 << (4 * (k % 2))                                          # 1.0
        b = torch.full((N, K // 2), 0x22, dtype=torch.uint8, device="cuda")
        sa = (120 + (torch.arange(M, device="cuda")[:, None] * 3 + torch.arange(34, device="cuda")) % 14).to(torch.uint8)
        sb = (115 + (torch.arange(N, device="cuda")[:, None] * 5 + 3 * torch.arange(34, device="cuda")) % 19).to(torch.uint8)
        pad = lambda t, n: torch.nn.functional.pad(t, (0, n - t.shape[1]))[:, :t.shape[1]]      # noqa: E731
        a, b, sa, sb = pad(a, 544), pad(b, 544), pad(sa, 48), pad(sb, 48)
        c = pkg.asgd_product4(a.view(torch.float4_e2m1fn_x2), sa.view(torch.float8_e8m0fnu), b.view(torch.float4_e2m1fn_x2), sb.view(torch.float8_e8m0fnu), out_dtype=F32)
        want = torch.exp2(sa[:, k // 32].double() - 127)[:, None] * torch.exp2(sb[:, k // 32].double() - 127)
        assert torch.equal(c.double(), want), k
    pkg.asgd_experts_sync()


def test_product4_without_inner_dimension_or_rows():
    q, s = torch.zeros(5, 0, dtype=torch.uint8, device="cuda").view(torch.float4_e2m1fn_x2), torch.zeros(5, 0, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    c = pkg.asgd_product4(q, s, q, s, out=torch.full((5, 5), 7.0, device="cuda"))
    assert (c == 0).all()
    a, sa = _operand(4, 256, 1)
    assert pkg.asgd_product4(a[:0], sa[:0], a, sa).shape == (0, 4)
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("M, N", [(150, 300), (1200, 2500)])
def test_product4_strides(M, N):
    a, sa = _operand(M, 512, 1)
    b, sb = _operand(N, 512, 2)
    want = pkg.asgd_product4(a, sa, b, sb, out_dtype=F32)
    big = torch.zeros(2 * M, 400, dtype=torch.uint8, device="cuda")
    big[::2, 16:272] = a.view(torch.uint8)
    scales = torch.full((2 * M, 64), 255, dtype=torch.uint8, device="cuda")
    scales[::2, 32:48] = sa.view(torch.uint8)
    out = torch.full((M, N + 33), -1.0, device="cuda")
    got = pkg.asgd_product4(big[::2, 16:272].view(a.dtype), scales[::2, 32:48].view(sa.dtype), b, sb, out=out[:, 1:N + 1])
    assert torch.equal(got, want) and (out[:, 0] == -1).all() and (out[:, N + 1:] == -1).all()
    with pytest.raises(binding.AsgdError):
        pkg.asgd_product4(big[::2, 8:264].view(a.dtype), sa, b, sb)                # rows that start between 16 bytes
    with pytest.raises(binding.AsgdError):
        pkg.asgd_product4(a, scales[::2, 8:24].view(sa.dtype), b, sb)
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("loads, N, K, out", [
    ([3, 0, 1, 16, 17, 0, 0, 40], 200, 300, F32), ([0] * 7 + [5], 256, 512, BF), ([100, 300, 0, 7, 513], 700, 1100, F32), ([1] * 64, 384, 640, F32),
    ([700, 0, 900, 3, 256, 255, 257, 1], 2240, 320, F32), ([2] * 300, 130, 64, F16)])
@pytest.mark.parametrize("first", [0, 3])
def test_product4_of_groups(loads, N, K, out, first):
    offsets = torch.tensor([first] + loads).cumsum(0).to(torch.int32).cuda()
    M, G = first + sum(loads) + 5, len(loads)
    a, sa = _operand(M, K, 3)
    b, sb = _operand(N, K, 4, (G,))
    c = torch.full((M, N), -7.0, device="cuda", dtype=out)
    pkg.asgd_product4(a, sa, b, sb, offsets=offsets, out=c)
    pkg.asgd_experts_sync()
    assert (c[:first] == -7).all() and (c[M - 5:] == -7).all()                     # rows of no group stay
    at = offsets.tolist()
    for g in range(G):
        if at[g] < at[g + 1]:
            r = slice(at[g], at[g + 1])
            _check_product(c[r], _values64(a[r], sa[r]), _values64(b[g], sb[g]), out)


@pytest.mark.parametrize("N, K", [(2744, 2080), (1300, 600), (1024, 200), (2300, 5130), (700, 130)])
def test_products_of_many_tiles_and_any_number_of_blocks(N, K):
    # tile after tile through every block, with odd and even numbers of K blocks and units, loads that differ
    loads = [700, 3, 0, 1200, 256, 511, 90, 2000, 1, 1300, 800, 640]
    offsets = torch.tensor([0] + loads).cumsum(0).to(torch.int32).cuda()
    a, sa = _operand(sum(loads), K, 3)
    b, sb = _operand(N, K, 4, (len(loads),))
    c = pkg.asgd_product4(a, sa, b, sb, offsets=offsets, out_dtype=F32)
    pkg.asgd_experts_sync()
    at = offsets.tolist()
    for g in range(len(loads)):
        r = slice(at[g], at[g + 1])
        if loads[g]:
            _check_product(c[r], _values64(a[r], sa[r]), _values64(b[g], sb[g]), F32)
    for _ in range(5):
        assert torch.equal(c, pkg.asgd_product4(a, sa, b, sb, offsets=offsets, out_dtype=F32))
    pkg.asgd_experts_sync()


def test_a_nan_scale_stays_in_its_row():
    for M, N in ((6, 300), (600, 2300)):
        a, sa = _operand(M, 640, 5)
        b, sb = _operand(N, 640, 6)
        want = pkg.asgd_product4(a, sa, b, sb, out_dtype=F32)
        sa2, sb2 = sa.view(torch.uint8).clone(), sb.view(torch.uint8).clone()
        sa2, sb2 = torch.nn.functional.pad(sa2, (0, 12))[:, :20], torch.nn.functional.pad(sb2, (0, 12))[:, :20]
        sa2[3, 7], sb2[150, 19] = 255, 255
        got = pkg.asgd_product4(a, sa2.view(sa.dtype), b, sb2.view(sb.dtype), out_dtype=F32)
        nan = torch.zeros_like(got, dtype=torch.bool)
        nan[3], nan[:, 150] = True, True
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


def test_quantize_and_multiply_as_a_layer_does():
    # tokens into their experts' order, 4 bits, every expert's matrix, back into token order
    T, E, top_k, D, N = 300, 8, 2, 448, 320
    g = _gen(11)
    x = torch.randn(T, D, generator=g, device="cuda").to(BF)
    w = torch.randn(E, N, D, generator=g, device="cuda") / D ** 0.5
    ids, weights, offsets, rows, source = pkg.asgd_route(torch.randn(T, E, generator=g, device="cuda"), top_k, align=16)
    wq, ws = zip(*(pkg.asgd_quantize4(m) for m in w))
    pack = lambda ts: torch.stack([torch.nn.functional.pad(t.view(torch.uint8), (0, -t.shape[1] % 16)) for t in ts])      # noqa: E731
    wq, ws = pack(wq)[..., :D // 2].view(torch.float4_e2m1fn_x2), pack(ws)[..., :D // 32].view(torch.float8_e8m0fnu)
    xq, xs = pkg.asgd_quantize4(x, source=source, per_token=top_k)
    z = pkg.asgd_product4(xq, xs, wq, ws, offsets=offsets, out_dtype=F32)
    y = pkg.asgd_combine(z, rows, weights)
    pkg.asgd_experts_sync()
    xv = pkg.asgd_dequantize4(*pkg.asgd_quantize4(x), dtype=F32).double()
    wv = torch.stack([_values64(q, s) for q, s in zip(wq, ws)])
    each = torch.einsum("td,end->ten", xv, wv).gather(1, ids.long()[..., None].expand(T, top_k, N))
    size = torch.einsum("td,end->ten", xv.abs(), wv.abs()).gather(1, ids.long()[..., None].expand(T, top_k, N))
    want = (each * weights.double()[..., None]).sum(1)
    bound = ((2 * (D + 8) + 4) * U * 1.01 * size * weights.double()[..., None]).sum(1)
    assert bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("M, N, K", [(5, 512, 1024), (20, 300, 4096), (700, 2300, 2048), (3000, 4000, 600)])
@pytest.mark.parametrize("limit, withhold", [(2000, True), (1, False), (30, False)])
def test_waits_given_up_leave_the_device_usable(M, N, K, limit, withhold):
    a, sa = _operand(M, K, 1)
    b, sb = _operand(N, K, 2)
    want = pkg.asgd_product4(a, sa, b, sb, out_dtype=F32)
    pkg.asgd_experts_sync()
    try:
        pkg.asgd_product_set_wait_drill(limit, withhold)
        pkg.asgd_product4(a, sa, b, sb, out_dtype=F32)
        if withhold:
            with pytest.raises(binding.AsgdError):
                pkg.asgd_experts_sync()
        else:
            try:
                pkg.asgd_experts_sync()
            except binding.AsgdError as e:
                assert e.status == binding.ASGD_ETIMEOUT
    finally:
        pkg.asgd_product_set_wait_drill()
    for _ in range(3):
        assert torch.equal(pkg.asgd_product4(a, sa, b, sb, out_dtype=F32), want)
    pkg.asgd_experts_sync()


def test_product4_replays_from_a_graph_on_another_stream():
    a, sa = _operand(40, 1024, 1)
    b, sb = _operand(600, 1024, 2)
    want = pkg.asgd_product4(a, sa, b, sb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.asgd_product4(a, sa, b, sb, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    x = _numbers(40, 1024, BF, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s = pkg.asgd_quantize4(x)
        c = pkg.asgd_product4(q, s, b, sb)
    x.copy_(_numbers(40, 1024, BF, 9))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c, pkg.asgd_product4(*pkg.asgd_quantize4(x), b, sb))
    pkg.asgd_experts_sync()
