"""The whole layer for a few tokens on the GPU against 64 bits.

Tolerances.  u = 2^-24.  The tokens' 8-bit values are those of asgd_quantize, the choice and the weights those the call returns (checked
against asgd_route).  A product's number is a sum of n terms within (min(n, 128) + 4 ceil(n / 128) + 8) u of the sum of their magnitudes (K blocks
on the tensor cores, scales, partial sums).  The activation carries that on by its slope and adds 8 u of itself.  Rounding the hidden
numbers to 8 bits is a step function: where the exact argument is farther from the middle between two 8-bit numbers than the kernel's argument can be from the
exact one, both round alike; where it is not, they may differ by one step.  What the second product makes of that, and its own
error, is summed with the weights.
"""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {F32: U, BF: 2.0 ** -8, F16: 2.0 ** -11}
SMALLEST = {F32: 2.0 ** -149, BF: 2.0 ** -133, F16: 2.0 ** -24}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrices(g, E, rows, K, fmt=E4):
    """[E, rows, K] in 8 bits (rows at multiples of 16 bytes) and the scales of 128 x 128 blocks."""
    parts = [pkg.asgd_quantize(torch.randn(rows, K, generator=g, device="cuda") / K ** 0.5, form="blocks", dtype=fmt) for _ in range(E)]
    ld = -(-K // 16) * 16
    q = torch.zeros(E, rows, ld, dtype=torch.uint8, device="cuda")
    for e, (p, _) in enumerate(parts):
        q[e, :, :K] = p.view(torch.uint8)
    return q[..., :K].view(fmt), torch.stack([s for _, s in parts])


def _values(q, s):
    rows, K = q.shape[-2:]
    return q.float().double() * s.double().repeat_interleave(128, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :K]


def _sum_u(n):
    return (min(n, 128) + 4 * -(-n // 128) + 8) * U


def _exact(x, w1, s1, w2, s2, ids, weights, act, dtype):
    """y in 64 bits [T, d] and how far the kernel's may be from it."""
    T, d = x.shape
    h = w2.shape[-1]
    gated = w1.shape[1] == 2 * h
    xq, xs = pkg.asgd_quantize(x)
    x64 = xq.float().double() * xs.double().repeat_interleave(128, 1)[:, :d]
    y, err = torch.zeros(T, d, dtype=torch.float64, device="cuda"), torch.zeros(T, d, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(y)
    for e in ids.unique().tolist():
        if e < 0:
            continue
        t, j = (ids == e).nonzero(as_tuple=True)
        A, B = _values(w1[e], s1[e]), _values(w2[e], s2[e])
        u, eu = x64[t] @ A.t(), _sum_u(d) * (x64[t].abs() @ A.abs().t())
        g, eg = u[:, :h], eu[:, :h]
        if act == "relu2":
            a = g.clamp_min(0).square()
            ea = 2 * g.clamp_min(0) * eg + eg.square() + 8 * U * a
        else:
            a = g * torch.sigmoid(g)
            ea = 1.11 * eg + 8 * U * a.abs()
        if gated:
            up, eup = u[:, h:], eu[:, h:]
            a, ea = a * up, ea * up.abs() + a.abs() * eup + ea * eup + U * (a * up).abs()
        # 8 bits: by blocks of 128
        pad = lambda v: torch.nn.functional.pad(v, (0, -h % 128)).unflatten(1, (-1, 128))      # noqa: E731
        av, ev = pad(a), pad(ea)
        m = av.abs().amax(2, keepdim=True).clamp_min(2.0 ** -100)
        off = ev.amax(2, keepdim=True) / m + 8 * U                     # relative error of the block's largest number
        arg = av * 448 / m
        earg = (ev * 448 / m + arg.abs() * off) * 1.01
        q = arg.float().to(E4).double()
        exponent = torch.floor(torch.log2(arg.abs().clamp_min(2.0 ** -6))).clamp_min(-6)
        step = torch.exp2(exponent - 3)
        # how far the argument is from the nearest middle between two neighbours (of either side's step)
        ratio = arg.abs() / step
        to_middle = (ratio - torch.floor(ratio) - 0.5).abs() * step
        unclear = to_middle <= earg
        scale = m / 448
        eq = q.abs() * scale * off + torch.where(unclear, 2 * step * scale, torch.zeros_like(step)) * (1 + off)
        flat = lambda v: v.flatten(1)[:, :h]                                                    # noqa: E731
        hv, eh = flat(q * scale), flat(eq)
        z, ez = hv @ B.t(), eh @ B.abs().t() + _sum_u(h) * ((hv.abs() + eh) @ B.abs().t())
        w = weights[t, j].double()[:, None]
        y.index_add_(0, t, w * z)
        err.index_add_(0, t, w.abs() * ez)
        size.index_add_(0, t, w.abs() * z.abs())
    err = err + (ids.shape[1] + 1) * U * (size + err)
    return y, err + HALF_STEP[dtype] * (y.abs() + err) + SMALLEST[dtype]


def _check(x, w1, s1, w2, s2, got, act, min_tight=True):
    y, ids, weights = got
    want, bound = _exact(x, w1, s1, w2, s2, ids.long(), weights, act, x.dtype)
    assert y.shape == x.shape and y.dtype == x.dtype and not torch.isnan(y).any()
    off = (y.double() - want).abs() - bound
    assert float(off.max()) <= 0.0, float(off.max())
    if min_tight and float(want.norm()) > 0:                           # the bound says something
        assert float(bound.norm()) < 0.5 * float(want.norm())


SHAPES = [
    # T, E, top_k, d, h, gated, act, type, score, groups, router, formats
    (1, 1, 1, 1, 1, False, "relu2", F32, "softmax", 1, None, (E4, E4)),
    (1, 4, 2, 16, 16, True, "silu", BF, "softmax", 1, None, (E4, E4)),
    (1, 128, 8, 2048, 768, True, "silu", BF, "softmax", 1, F32, (E4, E4)),
    (8, 256, 8, 512, 384, True, "silu", BF, "sigmoid", 8, None, (E4, E4)),
    (5, 40, 6, 130, 70, True, "relu2", F32, "sigmoid", 4, BF, (E4, E5)),
    (3, 600, 8, 200, 131, True, "silu", F16, "softmax", 1, F16, (E5, E4)),
    (60, 32, 4, 1040, 712, False, "relu2", F16, "sigmoid", 1, BF, (E4, E4)),
    (100, 16, 2, 384, 512, False, "silu", BF, "softmax", 1, None, (E4, E4)),
    (128, 8, 8, 256, 128, True, "silu", F32, "softmax", 1, F32, (E4, E4)),
    (128, 1000, 1, 128, 256, False, "relu2", F32, "sigmoid", 1, None, (E4, E4)),
    (33, 4, 3, 2304, 65, True, "relu2", BF, "softmax", 1, F32, (E4, E4)),
    (17, 64, 32, 300, 300, True, "silu", F32, "sigmoid", 1, None, (E4, E4)),
    (2, 3, 2, 4000, 2000, True, "silu", F32, "softmax", 1, F32, (E4, E4)),
    # where the blocks begin to share the choices out, and around 32 assignments
    (30, 12, 3, 384, 256, True, "silu", BF, "sigmoid", 3, F32, (E4, E4)),
    (31, 12, 3, 384, 256, False, "relu2", BF, "softmax", 1, None, (E4, E4)),
    (31, 40, 1, 256, 130, True, "silu", F32, "softmax", 1, F32, (E4, E4)),
    (32, 40, 1, 256, 130, False, "relu2", F32, "sigmoid", 1, None, (E4, E4)),
    (33, 40, 1, 256, 130, True, "relu2", F16, "softmax", 1, F16, (E4, E4)),
]


def _case(T, E, top_k, d, h, gated, act, dtype, score, groups, router, formats, seed=1):
    g = _gen(seed)
    x = (torch.randn(T, d, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(T, 1, generator=g, device="cuda"))).to(dtype)
    w1, s1 = _matrices(g, E, h * (2 if gated else 1), d, formats[0])
    w2, s2 = _matrices(g, E, d, h, formats[1])
    kw = dict(activation=act, score=score, groups=groups, groups_kept=(groups + 1) // 2, group_top=2 if groups > 1 else 1, scale=2.5,
              bias=torch.randn(E, generator=g, device="cuda") * 0.1 if score == "sigmoid" else None)
    if router is None:
        kw["logits"] = torch.randn(T, E, generator=g, device="cuda") * 1.5
    else:
        kw.update(router=(torch.randn(E, d, generator=g, device="cuda") / d ** 0.5).to(router), shift=torch.randn(E, generator=g, device="cuda") * 0.3, temperature=1.25)
    return (x, w1, s1, w2, s2, top_k), kw


ROUTE = ("score", "bias", "groups", "groups_kept", "group_top", "scale")


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(v).replace("torch.", "") for v in s[:7]))
def test_layer(shape):
    args, kw = _case(*shape)
    x, w1, s1, w2, s2, top_k = args
    got = pkg.asgd_expert_layer(*args, choice=True, **kw)
    pkg.asgd_experts_sync()
    y, ids, weights = got
    if kw.get("logits") is not None:
        want_ids, want_weights = pkg.asgd_route(kw["logits"], top_k, plan=False, **{k: kw[k] for k in ROUTE})
        assert torch.equal(ids, want_ids)
        assert float((weights - want_weights).abs().max()) <= 64 * U * 2.5        # sums of scores in another order
    else:
        logits = (x.double() @ kw["router"].double().t() - kw["shift"].double()) * kw["temperature"]
        want_ids, want_weights = pkg.asgd_route(logits.float(), top_k, plan=False, **{k: kw[k] for k in ROUTE})
        size = (x.double().abs() @ kw["router"].double().abs().t()).amax(1, keepdim=True) * kw["temperature"]
        same = (ids == want_ids).all(1)                                            # all but tokens whose choice hangs on the last bits
        assert int((~same).sum()) <= 1
        tol = (x.shape[1] * U * size + 64 * U) * 2.5 * 2                           # a score's slope is below 1; the renormalising sum doubles it
        assert bool(((weights - want_weights).abs() <= tol)[same].all())
    _check(x, w1, s1, w2, s2, got, kw["activation"])
    for _ in range(3):                                                             # no sum depends on timing
        assert torch.equal(pkg.asgd_expert_layer(*args, **kw), y)
    pkg.asgd_experts_sync()


def test_the_layer_is_what_the_separate_operators_give():
    # one chain of seven calls; what differs is the roundings between them (bf16 results of products: half a step of 2^-8 twice, through 8 bits)
    args, kw = _case(40, 16, 2, 512, 256, False, "relu2", F32, "sigmoid", 1, None, (E4, E4), seed=4)
    x, w1, s1, w2, s2, top_k = args
    y = pkg.asgd_expert_layer(*args, **kw)
    ids, weights, offsets, rows, source = pkg.asgd_route(kw["logits"], top_k, **{k: kw[k] for k in ROUTE})
    xq, xs = pkg.asgd_quantize(x, source=source, per_token=top_k)
    u = pkg.asgd_product(xq, xs, w1, s1, offsets=offsets, out_dtype=F32)
    hq, hs = pkg.asgd_quantize(torch.relu(u).square())
    z = pkg.asgd_product(hq, hs, w2, s2, offsets=offsets, out_dtype=F32)
    want = pkg.asgd_combine(z, rows, weights)
    # fp32 throughout: they differ in the order of sums, and by an 8-bit step where that decides a rounding (2^-4 of one of 256 hidden numbers)
    assert float((y - want).norm() / want.norm()) < 2.0 ** -8


@pytest.mark.parametrize("T, E, top_k, groups, kept", [(5, 300, 8, 1, 1), (7, 1000, 32, 1, 1), (16, 64, 4, 1, 1), (8, 96, 7, 6, 3), (40, 512, 16, 8, 8), (100, 33, 3, 11, 5), (2, 32, 32, 1, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", ["ties", "gone", "all equal"])
def test_choices_with_ties_and_unavailable_experts_are_those_of_the_routing(T, E, top_k, groups, kept, score, kind):
    g = _gen(T + E)
    logits = torch.randn(T, E, generator=g, device="cuda")
    if kind == "ties":
        logits = torch.round(logits * 2) / 2
    elif kind == "all equal":
        logits = torch.zeros(T, E, device="cuda")
    else:
        logits[torch.rand(T, E, generator=g, device="cuda") < 0.97] = -math.inf
    d, h = 16, 16
    w1, s1 = _matrices(g, 1, h, d)
    w2, s2 = _matrices(g, 1, d, h)
    many = lambda t: t.expand(E, *t.shape[1:]).contiguous() if t.dtype == F32 else t.view(torch.uint8).expand(E, *t.shape[1:]).contiguous().view(t.dtype)      # noqa: E731
    x = torch.randn(T, d, generator=g, device="cuda")
    kw = dict(score=score, groups=groups, groups_kept=kept, group_top=1, scale=1.5)
    want_ids, want_weights = pkg.asgd_route(logits, top_k, plan=False, **kw)
    y, ids, weights = pkg.asgd_expert_layer(x, many(w1), many(s1), many(w2), many(s2), top_k, logits=logits, choice=True, **kw)
    pkg.asgd_experts_sync()
    assert torch.equal(ids, want_ids)
    if score == "sigmoid":                                                         # (a softmax without any logit above -inf is NaN)
        assert float((weights - want_weights).abs().max()) <= 64 * U * 1.5
        _check(x, many(w1), many(s1), many(w2), many(s2), (y, ids, weights), "relu2", min_tight=False)


def test_layer_of_nothing_and_unavailable_experts():
    args, kw = _case(4, 8, 3, 256, 128, True, "silu", F32, "softmax", 1, None, (E4, E4))
    x, w1, s1, w2, s2, top_k = args
    empty = pkg.asgd_expert_layer(x[:0], *args[1:], **{**kw, "logits": kw["logits"][:0]})
    assert empty.shape == (0, 256)
    logits = kw["logits"].clone()
    logits[1] = -math.inf                                                          # no expert at all
    logits[2, 1:] = -math.inf                                                      # one
    got = pkg.asgd_expert_layer(*args, choice=True, **{**kw, "logits": logits, "score": "sigmoid"})
    assert (got[1][1] == -1).all() and (got[1][2] == torch.tensor([0, -1, -1], device="cuda")).all() and (got[0][1] == 0).all()
    _check(x, w1, s1, w2, s2, got, "silu")
    none = pkg.asgd_expert_layer(*args, **{**kw, "logits": torch.full_like(logits, -math.inf), "score": "sigmoid"})
    assert (none == 0).all()
    pkg.asgd_experts_sync()


def test_a_nan_stays_in_its_token():
    args, kw = _case(6, 8, 2, 256, 128, True, "silu", F32, "softmax", 1, None, (E4, E4))
    x = args[0].clone()
    want = pkg.asgd_expert_layer(*args, **kw)
    x[3, 100] = math.nan
    x[4, 7] = math.inf
    got = pkg.asgd_expert_layer(x, *args[1:], **kw)
    assert torch.isnan(got[3]).all() and torch.isnan(got[4]).any()
    keep = [0, 1, 2, 5]
    assert torch.equal(got[keep], want[keep])


def test_layer_strides():
    args, kw = _case(20, 12, 2, 200, 150, True, "silu", BF, "softmax", 1, F32, (E4, E4))
    x, w1, s1, w2, s2, top_k = args
    want = pkg.asgd_expert_layer(*args, **kw)
    bigx = torch.full((40, 333), math.nan, device="cuda", dtype=BF)
    bigx[::2, 3:203] = x
    bigr = torch.full((12, 401), math.nan, device="cuda")
    bigr[:, 1:201] = kw["router"]
    big1 = torch.zeros(12, 310, 320, dtype=torch.uint8, device="cuda")
    big1[:, :300, 32:232] = w1.view(torch.uint8)
    big2 = torch.zeros(24, 200, 160, dtype=torch.uint8, device="cuda")
    big2[::2, :, :150] = w2.view(torch.uint8)
    bs1 = torch.full((12, 2, 7), math.nan, device="cuda").permute(0, 2, 1)         # columns of blocks first
    bs1[:, :3, :] = s1
    got = pkg.asgd_expert_layer(bigx[::2, 3:203], big1[:, :300, 32:232].view(E4), bs1[:, :3, :], big2[::2, :, :150].view(E4), s2, top_k,
                                **{**kw, "router": bigr[:, 1:201]})
    # the router's sum runs over the same numbers, read four at a time or one by one
    assert torch.equal(got, want)
    logits = torch.randn(20, 30, device="cuda").to(F16)
    kw = {k: v for k, v in kw.items() if k not in ("router", "shift", "temperature")}
    a = pkg.asgd_expert_layer(*args, **kw, logits=logits[:, 9:21])
    assert torch.equal(a, pkg.asgd_expert_layer(*args, **kw, logits=logits[:, 9:21].contiguous()))
    with pytest.raises(binding.AsgdError):
        pkg.asgd_expert_layer(x, big1[:, :300, 8:208].view(E4), s1, w2, s2, top_k, logits=logits[:, :12], activation="silu")
    pkg.asgd_experts_sync()


def test_layer_in_a_graph_and_on_several_streams():
    args, kw = _case(8, 32, 4, 512, 256, True, "silu", BF, "softmax", 1, F32, (E4, E4))
    x = args[0]
    want = pkg.asgd_expert_layer(*args, **kw)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [pkg.asgd_expert_layer(*args, **kw, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = pkg.asgd_expert_layer(*args, **kw)
        second = pkg.asgd_expert_layer(first, *args[1:], **kw)
    x.copy_(torch.randn(8, 512, device="cuda"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    one = pkg.asgd_expert_layer(*args, **kw)
    assert torch.equal(first, one) and torch.equal(second, pkg.asgd_expert_layer(one, *args[1:], **kw))
    pkg.asgd_experts_sync()


def test_graphs_replayed_at_once_on_several_streams_beside_products():
    """Layers of several streams, each of which wants all SMs, and products that hold some of them."""
    cases = [_case(8, 32, 4, 512, 256, True, "silu", BF, "softmax", 1, F32, (E4, E4)), _case(40, 16, 4, 384, 200, False, "relu2", F16, "sigmoid", 1, None, (E4, E4))]
    a = torch.randn(700, 1024, generator=_gen(5), device="cuda", dtype=BF)
    w = pkg.asgd_quantize4(torch.randn(2048, 1024, generator=_gen(6), device="cuda", dtype=BF))
    calls = [lambda args=args, kw=kw: pkg.asgd_expert_layer(*args, **kw) for args, kw in cases] + [lambda: pkg.asgd_product4(*pkg.asgd_quantize4(a), *w)]
    want = [call() for call in calls]
    graphs, got = [], []
    for call in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append([call() for _ in range(8)])
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, v) for v, gs in zip(want, got) for g in gs)
    pkg.asgd_experts_sync()


@pytest.mark.parametrize("T, router", [(1, None), (30, F32)])
@pytest.mark.parametrize("limit, withhold", [(2000, True), (1, False), (40, False)])
def test_waits_given_up_leave_the_device_usable(T, router, limit, withhold):
    args, kw = _case(T, 16, 2, 1024, 512, True, "silu", BF, "softmax", 1, router, (E4, E4))
    want = pkg.asgd_expert_layer(*args, **kw)
    pkg.asgd_experts_sync()
    try:
        pkg.asgd_product_set_wait_drill(limit, withhold)
        pkg.asgd_expert_layer(*args, **kw)
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
        assert torch.equal(pkg.asgd_expert_layer(*args, **kw), want)
    pkg.asgd_experts_sync()


def test_the_trained_layer_serves_what_it_computes_in_training():
    from paper_1505_04956_b200 import expert_layer
    X, target = expert_layer.make_task(600, 128, 4, seed=7)
    layer = expert_layer.make_layer(X, 4, 256, seed=7)
    for _ in range(3):
        layer.step(X, target, 0.5)
    want, _ = layer.forward(X[:100])
    got = layer.serve(X[:100], layer.eight_bits())
    pkg.asgd_experts_sync()
    # forward() rounds the first products to bf16 (half a step of 2^-8, doubled by the square) before they are rounded to 8 bits, whose step of 2^-4
    # a twelfth to a sixth of them then crosses: 2^-4 / sqrt(6) of such numbers is 2.6 %
    assert torch.equal(got, layer.serve(X[:100])) and float((got - want).norm() / want.norm()) < 0.05
