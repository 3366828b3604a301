"""The norm of many gradients and clipping on the GPU against 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32.  Squares of fp32, bf16 and fp16 numbers are exact in fp64 (48 bits of 53), and the sum of
n <= 2^30 of them is within 2^-23 of itself relatively (2^30 * 2^-53), so the root is within 2^-24 + the rounding to fp32 u: 2 u covers
the norm.  The factor is a quotient of the norm plus 1e-6 (three roundings: 3 u, and the norm's 2 u), the product one more, and a result is
rounded to its type by half a step at most, or by half of the type's smallest number.
"""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_STEP = {F32: U, BF: 2.0 ** -8, F16: 2.0 ** -11}
SMALLEST = {F32: 2.0 ** -149, BF: 2.0 ** -133, F16: 2.0 ** -24}


def _norm64(ts):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in ts))


def _tensors(seed, sizes, types, scale=1.0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = torch.randn(n + offset, generator=g, device="cuda") * (scale * (1 + i % 3))
        out.append(t.to(types[i % len(types)])[offset:])
    return out


def _check(ts, max_norm, norm, got):
    want = _norm64(ts)
    assert abs(float(norm) - want) <= 2 * U * want
    f = min(1.0, max_norm / (want + 1e-6))
    for t, o in zip(ts, got):
        exact = t.double() * f
        bound = exact.abs() * (6 * U + HALF_STEP[t.dtype]) + SMALLEST[t.dtype]
        assert o.dtype == t.dtype and o.shape == t.shape
        assert bool(((o.double() - exact).abs() <= bound).all())


CASES = [
    ([1], [F32]), ([5], [BF]), ([7, 0, 9], [F16]), ([16384], [F32]), ([16385, 3, 1, 1, 70001], [F32, BF, F16]),
    ([1023, 1025] * 40, [BF, F32]), (list(range(1, 700)), [F16, F32, BF]), ([64] * 1300 + [1 << 20], [F32]), ([3_000_001], [BF]), ([5_000_003, 17, 2_000_000], [F16, F32]),
]


@pytest.mark.parametrize("sizes, types", CASES)
@pytest.mark.parametrize("offset", [0, 1, 4, 13])
def test_norm_and_clipping(sizes, types, offset):
    ts = _tensors(len(sizes), sizes, types, 0.1, offset)
    for max_norm in (0.25, 1e9):
        out = [torch.full_like(t, 7.0) for t in ts]
        keep = [t.clone() for t in ts]
        norm = pkg.asgd_clip_grads(ts, max_norm, out=out)
        assert norm.shape == () and norm.dtype == F32
        _check(ts, max_norm, norm, out)
        assert all(torch.equal(a, b) for a, b in zip(ts, keep))
        assert torch.equal(pkg.asgd_grad_norm(ts), norm)
        assert torch.equal(pkg.asgd_clip_grads(ts, max_norm), norm)       # in place: the same numbers
        assert all(torch.equal(a, b) for a, b in zip(ts, out))
        for t, k in zip(ts, keep):
            t.copy_(k)


def test_numbers_around_a_tensor_stay():
    base = torch.ones(3 * 1001, device="cuda", dtype=BF)
    t = base[1001:2002]
    pkg.asgd_clip_grads([t], 0.5)
    assert bool((base[:1001] == 1).all()) and bool((base[2002:] == 1).all()) and bool((t < 1).all())


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_views_of_one_buffer(dtype):
    # neighbours in memory that begin anywhere, in place and into a buffer that begins elsewhere
    sizes = [1, 2, 3, 5, 8, 13, 40, 1000, 100_001, 7, 4096]
    flat = torch.randn(sum(sizes) + 9, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
    for first in (0, 1, 5):
        at = [first + sum(sizes[:i]) for i in range(len(sizes))]
        ts = [flat[a:a + n] for a, n in zip(at, sizes)]
        keep = flat.clone()
        room = torch.full((sum(sizes) + 9,), 7.0, device="cuda", dtype=dtype)
        out = [room[a + 2:a + 2 + n] for a, n in zip(at, sizes)]
        norm = pkg.asgd_clip_grads(ts, 0.5, out=out)
        _check(ts, 0.5, norm, out)
        assert bool((room[:first + 2] == 7).all()) and bool((room[first + 2 + sum(sizes):] == 7).all()) and torch.equal(flat, keep)
        pkg.asgd_clip_grads(ts, 0.5)
        assert all(torch.equal(a, b) for a, b in zip(ts, out))
        assert torch.equal(flat[:first], keep[:first]) and torch.equal(flat[first + sum(sizes):], keep[first + sum(sizes):])
        flat.copy_(keep)


def test_no_numbers():
    for ts in ([], [torch.empty(0, device="cuda")], [torch.empty(0, 5, device="cuda", dtype=BF)] * 3):
        assert float(pkg.asgd_grad_norm(ts)) == 0.0
        assert float(pkg.asgd_clip_grads(ts, 1.0)) == 0.0


def test_squares_beyond_the_range_of_32_bits():
    big, small = torch.full((1000,), 1e30, device="cuda"), torch.full((1000,), 1e-30, device="cuda")
    for ts in ([big], [small]):
        want = _norm64(ts)
        assert abs(float(pkg.asgd_grad_norm(ts)) - want) <= 2 * U * want
    ts = [big.clone()]
    norm = pkg.asgd_clip_grads(ts, 1.0)
    _check([big], 1.0, norm, ts)
    assert float(pkg.asgd_grad_norm([torch.full((100,), 3e38, device="cuda")])) == math.inf


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_infinities_and_nans(dtype):
    x = torch.randn(5000, device="cuda").to(dtype)
    x[77] = math.inf
    other = torch.ones(3000, device="cuda")
    ts = [x, other]
    assert float(pkg.asgd_clip_grads(ts, 1.0)) == math.inf
    assert math.isnan(float(x[77])) and float(x[:77].abs().sum()) == 0 and float(other.abs().sum()) == 0
    x = torch.randn(5000, device="cuda").to(dtype)
    keep = x.clone()
    x[4999] = math.nan
    assert math.isnan(float(pkg.asgd_clip_grads([x], math.inf)))
    assert torch.equal(x[:4999], keep[:4999])                       # without a limit nothing is scaled
    assert math.isnan(float(pkg.asgd_clip_grads([x, other], 1.0)))
    assert bool(x.isnan().all()) and bool(other.isnan().all())


def test_results_do_not_depend_on_timing_and_a_graph_replays():
    ts = _tensors(3, [100_003, 5, 2_000_001], [BF, F32, F32])
    out = [torch.empty_like(t) for t in ts]
    first = pkg.asgd_clip_grads(ts, 0.1, out=out)
    for _ in range(5):
        assert torch.equal(pkg.asgd_grad_norm(ts), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = [torch.empty_like(t) for t in ts]
    pkg.asgd_clip_grads(ts, 0.1, out=again, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = pkg.asgd_clip_grads(ts, 0.1, out=again)
    for t in ts:
        t.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    _check(ts, 0.1, norm, again)


def test_neighbours_and_inputs_that_share_memory():
    buffer = torch.randn(1000, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    before = buffer.clone()
    out = torch.empty(2, 600, device="cuda")
    norm = pkg.asgd_clip_grads([buffer[:600], buffer[400:]], 1.0, out=[out[0], out[1]])
    factor = 1.0 / (math.sqrt((before[:600].double() ** 2).sum() + (before[400:].double() ** 2).sum()) + 1e-6)
    for got, x in ((out[0], before[:600]), (out[1], before[400:])):
        assert ((got.double() - x.double() * factor).abs() <= 6 * U * (x.double() * factor).abs() + SMALLEST[F32]).all()
    assert torch.equal(buffer, before)
    assert torch.equal(pkg.asgd_clip_grads([buffer[600:], buffer[:600]], 1e9), pkg.asgd_grad_norm([before[600:], before[:600]]))
    with pytest.raises(pkg.AsgdError):
        pkg.asgd_clip_grads([buffer[:600], buffer[599:]], 1.0)
    assert torch.equal(buffer, before) and float(norm) > 1


def test_refusals():
    x = torch.ones(10, device="cuda")
    for bad in ([x, x], [x[::2]], [x.double()], [x.cpu()], [x.int()]):
        with pytest.raises(ValueError):
            pkg.asgd_clip_grads(bad, 1.0)
    for out in ([], [torch.ones(9, device="cuda")], [x.bfloat16()], [x[::1], x]):
        with pytest.raises(ValueError):
            pkg.asgd_clip_grads([x], 1.0, out=out)
    with pytest.raises(ValueError):
        pkg.asgd_clip_grads([x, torch.ones(10, device="cuda")], 1.0, out=[x, x])


def test_a_clipped_step_of_the_layer_moves_by_the_clipped_gradients():
    from paper_1505_04956_b200 import expert_layer
    X, target = expert_layer.make_task(600, 128, 4, seed=5)
    layer = expert_layer.make_layer(X, 4, 256, seed=5)
    before = [t.clone() for t in (layer.router, layer.w1, layer.w2)]
    y, c = layer.forward(X)
    diff = y - target
    grads = [t.clone() for t in layer.gradients(X, diff * (2.0 / diff.numel()), c)[:3]]
    limit = 0.25 * _norm64(grads)
    layer.step(X, target, 0.5, max_norm=limit)
    f = limit / (_norm64(grads) + 1e-6)
    for b, after, g, rate in zip(before, (layer.router, layer.w1, layer.w2), grads, (0.025, 0.5, 0.5)):
        want = b.double() - rate * f * g.double()
        # the factor's 5 u, the product, the rate's two roundings, the difference's
        bound = 10 * U * (rate * f * g.double()).abs() + 2 * U * want.abs()
        assert bool(((after.double() - want).abs() <= bound).all())
