"""More operators of a layer of experts, as cases that can be timed and compared: microscaled 4-bit operands and their
products, a whole layer for a few tokens, and the global gradient norm with clipping.

With `own` false every operator is computed in its plain form (elementary torch operations in 32 bits, rounded once
at the end); with `own` true by the calls a user makes of the framework.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
E4M3 = torch.float8_e4m3fn
BLOCK = 128                                   # 8-bit numbers that share a scale
BLOCK4 = 32                                   # 4-bit numbers that share a power of two
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the gradients of a small layer of eight experts (router, two matrices each): one step of its training loop
        dict(name="clip, a small layer", op="clip", layers=1, experts=8, d=256, h=512, dtype="f32", max_norm=1.0),
        # the gradients of a stack of layers in 16 bits, far larger than the caches
        dict(name="clip, 14 layers", op="clip", layers=14, experts=4, d=1537, h=1999, dtype="bf16", max_norm=0.5),
        # the norm alone, for the log, over many tensors of mixed types and odd sizes
        dict(name="norm, 512 tensors", op="norm", layers=128, experts=1, d=333, h=1021, dtype="mixed", max_norm=0.0),
        # tokens gathered into their experts' order on the way to 4 bits, and what they then stand for
        dict(name="quantize4 into experts", op="quantize4", T=8192, D=4096, top_k=4, dtype="bf16", values="bf16"),
        # weights of odd sizes
        dict(name="quantize4, 4001 rows", op="quantize4", T=4001, D=2058, top_k=0, dtype="f32", values="f32"),
        # one serving step of five sequences through a dense layer: the weights' bytes
        dict(name="product4, 5 rows", op="product4", M=5, N=4096, K=4096, groups=0, out="bf16"),
        # a prompt through a large dense layer: the tensor pipe's rate
        dict(name="product4, 8192 rows", op="product4", M=8192, N=8192, K=8192, groups=0, out="bf16"),
        # a serving step through 64 experts, a handful of rows each and some with none: every expert's weights once
        dict(name="experts4, 256 rows", op="product4", M=256, N=2048, K=2048, groups=64, out="bf16"),
        # a batch through 32 experts of uneven load and odd sizes
        dict(name="experts4, 16384 rows", op="product4", M=16384, N=2744, K=2080, groups=32, out="f16"),
        # one token of one sequence through a layer of gated experts, its router included: latency, then the weights' bytes
        dict(name="layer, 1 token", op="layer", T=1, E=128, top_k=8, d=2048, h=768, gated=True, act="silu", score="softmax", groups=1,
             router="f32", dtype="bf16"),
        # a serving step of eight sequences, experts in groups chosen by sigmoid scores and a balance bias
        dict(name="layer, 8 tokens", op="layer", T=8, E=256, top_k=8, d=2048, h=512, gated=True, act="silu", score="sigmoid", groups=8,
             router="none", dtype="bf16"),
        # sixty tokens, several for every expert, in the form the framework trains (squared rectifier, no gate), odd sizes
        dict(name="layer, 60 tokens", op="layer", T=60, E=32, top_k=4, d=2064, h=1400, gated=False, act="relu2", score="sigmoid", groups=1,
             router="bf16", dtype="f16"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(step * -(-lo // step), min(v, hi // step * step))


def draw(rng):
    op = rng.choice(["clip", "norm", "quantize4", "quantize4", "product4", "product4", "product4", "layer", "layer", "layer"])
    if op in ("clip", "norm"):
        c = dict(op=op, layers=rng.randint(1, 14) if op == "clip" else _log(rng, 1, 200), experts=rng.choice([1, 1, 2, 8]), d=_log(rng, 16, 2048),
                 h=_log(rng, 16, 4096), dtype=rng.choice(["f32", "bf16", "f16", "mixed"]), max_norm=rng.choice([0.1, 1.0, 1e4]) if op == "clip" else 0.0)
        while c["layers"] > 1 and 2 * c["layers"] * c["experts"] * c["d"] * c["h"] > 150_000_000:
            c["layers"] //= 2
        return c
    if op == "quantize4":
        top_k = rng.choice([0, 0, 2, 4, 8])
        return dict(op=op, T=_log(rng, 1, 8192 if top_k < 8 else 4096), D=_log(rng, 32, 4096, rng.choice([1, 2, 32])), top_k=top_k,
                    dtype=rng.choice(["f32", "bf16", "f16"]), values=rng.choice(["f32", "bf16", "f16"]))
    if op == "product4":
        groups = rng.choice([0, 0, 8, 32, 64])
        return dict(op=op, M=_log(rng, 1, 16384 if groups else 8192), N=_log(rng, 256, 4096, 8), K=_log(rng, 256, 4096, rng.choice([2, 32, 128])),
                    groups=groups, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    score, groups = rng.choice(["softmax", "sigmoid"]), rng.choice([1, 1, 4])
    c = dict(op=op, T=_log(rng, 1, 128), E=groups * _log(rng, 8, 128 // groups), top_k=rng.randint(1, 8), d=_log(rng, 256, 4096, rng.choice([8, 128])),
             h=_log(rng, 128, 2048, rng.choice([8, 128])), gated=rng.random() < 0.6, act=rng.choice(["silu", "relu2"]), score=score, groups=groups,
             router=rng.choice(["none", "f32", "bf16"]), dtype=rng.choice(["bf16", "f16"]))
    while c["E"] > 8 * groups and 3 * c["E"] * c["d"] * c["h"] > 600_000_000:
        c["E"] = c["E"] // 2 // groups * groups
    return c


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _shapes(c):
    """The tensors of a stack of layers: router, bias of the choice, and the experts' two matrices."""
    of_layer = [(c["experts"], c["d"]), (c["experts"],), (c["experts"], c["h"], c["d"]), (c["experts"], c["d"], c["h"])]
    return of_layer * c["layers"]


def _types(c):
    n = len(_shapes(c))
    return ["f32", "bf16", "f16"] * n if c["dtype"] == "mixed" else [c["dtype"]] * n


def _power(x):
    """The power of two of every 32 neighbours of x [..., n, 32]: the smallest s with max|x| <= 6 s; x is finite."""
    m, e = torch.frexp(x.abs().amax(-1).clamp_min(2.0 ** -100))        # m in [1/2, 1)
    return torch.ldexp(torch.ones_like(m), e - 3 + (m > 0.75))


def _round4(v):
    """To the nearest of E2M1's numbers, ties to the even one; |v| <= 6."""
    a = v.abs()
    r = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2))
    return torch.copysign(r, v)


def _blocks4(x):
    """4-bit values of x [rows, K] (before their powers of two, [rows, blocks, 32]) and the powers [rows, blocks]."""
    v = torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK4)).unflatten(-1, (-1, BLOCK4))
    s = _power(v)
    return _round4(v / s[..., None]), s


def _operand4(g, shape):
    """A 4-bit operand [..., rows, K / 2] and its scales [..., rows, blocks] as a quantiser leaves them, rows at multiples of 16 bytes:
    numbers of unit variance, every 61st column ten times as large."""
    K = shape[-1]
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., ::61] *= 10
    v, s = _blocks4(x)
    v = v.flatten(-2)
    a = v.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * (v < 0).to(torch.uint8)
    q = code[..., 0::2] + 16 * code[..., 1::2]
    byte = (torch.frexp(s)[1] + 126).to(torch.uint8)

    def strided(t, n):
        ld = _ceil(n, 16) * 16
        store = torch.zeros(*t.shape[:-1], ld, dtype=torch.uint8, device="cuda")
        store[..., :n] = t[..., :n]
        return store[..., :n]
    return strided(q, _ceil(K, 2)).view(torch.float4_e2m1fn_x2), strided(byte, byte.shape[-1]).view(torch.float8_e8m0fnu)


def _loads(rng_cpu, groups, rows):
    """Rows per group: a skewed multinomial (popular and unpopular experts, some with nothing)."""
    p = torch.rand(groups, generator=rng_cpu).pow(2) + 0.01
    n = torch.multinomial(p, rows, replacement=True, generator=rng_cpu)
    return torch.bincount(n, minlength=groups)


def _weights8(g, E, rows, K):
    """Experts' matrices [E, rows, K] in 8 bits with the scales of their 128 x 128 blocks, rows at multiples of 16 bytes."""
    x = torch.randn(E, rows, K, generator=g, device="cuda") / K ** 0.5
    v = torch.nn.functional.pad(x, (0, -K % BLOCK, 0, -rows % BLOCK)).unflatten(2, (-1, BLOCK)).unflatten(1, (-1, BLOCK))
    amax = v.abs().amax((2, 4)).clamp_min(2.0 ** -100)
    q = (v * (448.0 / amax)[:, :, None, :, None]).flatten(3, 4).flatten(1, 2)[:, :rows, :K].to(E4M3)
    ld = _ceil(K, 16) * 16
    store = torch.zeros(E, rows, ld, dtype=torch.uint8, device="cuda")
    store[..., :K] = q.view(torch.uint8)
    return store[..., :K].view(E4M3), amax * (1.0 / 448.0)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.Generator().manual_seed(seed)
    s = dict(case)
    op = case["op"]
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")                      # noqa: E731
    if op in ("clip", "norm"):
        # the scale of gradients differs from tensor to tensor
        size = torch.exp(torch.randn(len(_shapes(case)), generator=c)).tolist()
        s["grads"] = [(randn(*shape) * (0.02 * k)).to(DTYPE[t]) for shape, t, k in zip(_shapes(case), _types(case), size)]
        s["out"] = [torch.empty_like(v) for v in s["grads"]] if op == "clip" else None
    elif op == "quantize4":
        x = randn(case["T"], case["D"]) * torch.exp(randn(case["T"], 1))
        x[:, ::67] *= 10
        s["x"] = x.to(DTYPE[case["dtype"]])
        s["source"] = torch.randperm(case["T"] * case["top_k"], generator=g, device="cuda").to(torch.int32) if case["top_k"] else None
    elif op == "product4":
        s["a"], s["a_scale"] = _operand4(g, (case["M"], case["K"]))
        s["b"], s["b_scale"] = _operand4(g, ((case["groups"],) if case["groups"] else ()) + (case["N"], case["K"]))
        s["offsets"] = None
        if case["groups"]:
            n = _loads(c, case["groups"], case["M"])
            s["most"] = int(n.max())
            s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).cuda()
    else:
        T, E, d, h = (case[k] for k in ("T", "E", "d", "h"))
        s["x"] = (randn(T, d) * torch.exp(0.5 * randn(T, 1))).to(DTYPE[case["dtype"]])
        s["w1"], s["w1_scale"] = _weights8(g, E, h * (2 if case["gated"] else 1), d)
        s["w2"], s["w2_scale"] = _weights8(g, E, d, h)
        s["bias"] = randn(E) * 0.1 if case["score"] == "sigmoid" else None
        pop = randn(E) * 0.5
        s["logits"] = s["matrix"] = s["shift"] = None
        if case["router"] == "none":
            s["logits"] = randn(T, E) * 1.5 + pop
        else:
            s["matrix"] = (randn(E, d) / d ** 0.5).to(DTYPE[case["router"]])
            s["shift"] = -pop
    return s


TEMPERATURE = 1.25                            # of the router's logits


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else PLAIN[s["op"]](s)


def _own(s):
    import paper_1505_04956_b200 as pkg
    op = s["op"]
    if op == "norm":
        return pkg.asgd_grad_norm(s["grads"])
    if op == "clip":
        return dict(norm=pkg.asgd_clip_grads(s["grads"], s["max_norm"], out=s["out"]), out=s["out"])
    if op == "quantize4":
        q, scale = pkg.asgd_quantize4(s["x"], source=s["source"], per_token=max(1, s["top_k"]))
        return pkg.asgd_dequantize4(q, scale, s["D"], dtype=DTYPE[s["values"]])
    if op == "product4":
        return pkg.asgd_product4(s["a"], s["a_scale"], s["b"], s["b_scale"], offsets=s["offsets"], out_dtype=DTYPE[s["out"]])
    return pkg.asgd_expert_layer(
        s["x"], s["w1"], s["w1_scale"], s["w2"], s["w2_scale"], s["top_k"], logits=s["logits"], router=s["matrix"], shift=s["shift"],
        temperature=TEMPERATURE, activation=s["act"], score=s["score"], bias=s["bias"], groups=s["groups"],
        groups_kept=(s["groups"] + 1) // 2, group_top=1 if s["groups"] == 1 else 2, renormalise=True, scale=2.5)


# ---- plain forms, 32 bits ----

def _norm(s):
    return torch.stack([v.double().square().sum() for v in s["grads"]]).sum().sqrt()      # long sums


def _plain_norm(s):
    return _norm(s).float()


def _plain_clip(s):
    norm = _norm(s).float()
    f = (s["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    return dict(norm=norm, out=[(v.float() * f).to(v.dtype) for v in s["grads"]])


def _plain_quantize4(s):
    x = s["x"].float()
    if s["source"] is not None:
        x = x[s["source"].long() // s["top_k"]]
    v, scale = _blocks4(x)
    return (v * scale[..., None]).flatten(-2)[:, :s["D"]].to(DTYPE[s["values"]])


def _values4(q, scale, K):
    """What a 4-bit operand stands for, in 32 bits."""
    q, byte = q.view(torch.uint8).long(), scale.view(torch.uint8).int()
    v = torch.tensor(E2M1, device=q.device)[torch.stack([q & 15, q >> 4], -1).flatten(-2)][..., :K]
    s = torch.ldexp(torch.ones(byte.shape, device=q.device), byte - 127)
    return v * s.repeat_interleave(BLOCK4, dim=-1)[..., :K]


def _plain_product4(s):
    a, b = _values4(s["a"], s["a_scale"], s["K"]), _values4(s["b"], s["b_scale"], s["K"])
    dt = DTYPE[s["out"]]
    if not s["groups"]:
        return (a @ b.t()).to(dt)
    M = s["M"]
    at = s["offsets"][:-1, None].long() + torch.arange(s["most"], device=a.device)
    at = torch.where(at < s["offsets"][1:, None], at, M)
    a = torch.cat([a, torch.zeros_like(a[:1])])
    y = torch.empty(M + 1, s["N"], device=a.device)
    y[at.reshape(-1)] = torch.bmm(a[at], b.transpose(1, 2)).reshape(-1, s["N"])
    return y[:M].to(dt)


def _eight(x):
    """What the rows of x stand for after a rounding to 8 bits with a scale for each 128 neighbours."""
    n = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    a = v.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    q = (v * (torch.full_like(a, 448.0) / a)).to(E4M3).to(x.dtype)
    return (q * (a * (1.0 / 448.0))).flatten(-2)[..., :n]


def _values8(q, scale):
    rows, K = q.shape[-2:]
    return q.float() * scale.repeat_interleave(BLOCK, dim=-2)[..., :rows, :].repeat_interleave(BLOCK, dim=-1)[..., :K]


def _plain_route(s, x):
    """ids and weights; every decision as the framework's routing takes it."""
    G, E = s["groups"], s["E"]
    if s["logits"] is not None:
        x = s["logits"].float()
    else:                                                              # in 64 bits: a choice may hang on the last one
        x = ((x.double() @ s["matrix"].double().t() - s["shift"]) * TEMPERATURE).float()
    if s["score"] == "sigmoid":
        p = torch.reciprocal(torch.exp(-x) + 1.0)
    else:
        e = torch.exp(x - x.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
    key = x if s["bias"] is None and G == 1 else p if s["bias"] is None else p + s["bias"]
    if G > 1:
        best = key.reshape(-1, G, E // G).sort(dim=2, descending=True).values
        kept = (best[..., 0] + best[..., 1]).sort(dim=1, descending=True, stable=True).indices[:, :(G + 1) // 2]
        out = torch.ones(key.shape[0], G, dtype=torch.bool, device=x.device).scatter(1, kept, False)
        key = key.masked_fill(out.repeat_interleave(E // G, dim=1), -math.inf)
    ids = key.sort(dim=1, descending=True, stable=True).indices[:, :s["top_k"]]
    w = p.gather(1, ids)
    return ids, 2.5 * w / (w.sum(1, keepdim=True) + 1e-20)


def _act(s, u):
    g, up = (u[..., :s["h"]], u[..., s["h"]:]) if s["gated"] else (u, 1.0)
    a = g * torch.reciprocal(torch.exp(-g) + 1.0) if s["act"] == "silu" else torch.relu(g) * torch.relu(g)
    return a * up


def _plain_layer(s):
    ids, w = _plain_route(s, s["x"])
    x = _eight(s["x"].float())
    T, K, E = s["T"], s["top_k"], s["E"]
    take = lambda q, i: q.view(torch.uint8)[i].view(E4M3)                                       # noqa: E731
    if T * K < E:                                                      # every assignment by its own expert
        i = ids.reshape(-1)
        rows = x.repeat_interleave(K, 0)[:, :, None]
        h = _eight(_act(s, torch.bmm(_values8(take(s["w1"], i), s["w1_scale"][i]), rows)[..., 0]))
        z = torch.bmm(_values8(take(s["w2"], i), s["w2_scale"][i]), h[..., None])[..., 0].reshape(T, K, -1)
        return (z * w[..., None]).sum(1).to(s["x"].dtype)
    h = _eight(_act(s, torch.matmul(x, _values8(s["w1"], s["w1_scale"]).transpose(1, 2))))      # every token by every expert
    z = torch.matmul(h, _values8(s["w2"], s["w2_scale"]).transpose(1, 2))                       # [E, T, d]
    z = z.transpose(0, 1).gather(1, ids[..., None].expand(T, K, s["d"]))
    return (z * w[..., None]).sum(1).to(s["x"].dtype)


PLAIN = dict(norm=_plain_norm, clip=_plain_clip, quantize4=_plain_quantize4, product4=_plain_product4, layer=_plain_layer)


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("clip", "norm"):
        n = sum(math.prod(shape) * SIZE[t] for shape, t in zip(_shapes(case), _types(case)))
        k = sum(math.prod(shape) for shape in _shapes(case))
        return dict(bytes=n * (2 if op == "clip" else 1), flops=k * (3 if op == "clip" else 2))
    if op == "quantize4":
        T, D = case["T"], case["D"]
        R = T * max(1, case["top_k"])
        return dict(bytes=T * D * SIZE[case["dtype"]] + R * (_ceil(D, 2) + _ceil(D, BLOCK4)) + R * D * SIZE[case["values"]] + (4 * R if case["top_k"] else 0),
                    flops=3 * R * D)
    if op == "product4":
        M, N, K, G = case["M"], case["N"], case["K"], case["groups"]
        row = _ceil(K, 2) + _ceil(K, BLOCK4)
        # weights of the experts that have rows, on average over the loads that _loads() draws
        used = sum(1 - math.exp(-M * (((i + 0.5) / 64) ** 2 + 0.01) / (G * (1 / 3 + 0.01))) for i in range(64)) / 64 * G if G else 1
        return dict(bytes=M * row + round(used * N * row) + M * N * SIZE[case["out"]], flops=2 * M * N * K)
    T, E, K, d, h = (case[k] for k in ("T", "E", "top_k", "d", "h"))
    numbers = (3 if case["gated"] else 2) * d * h
    used = E * (1 - (1 - K / E) ** T)                                  # experts in use, were all equally popular
    route = E * d * SIZE[case["router"]] + 4 * E if case["router"] != "none" else 4 * T * E
    return dict(bytes=round(used * (numbers + numbers / 4096)) + route + 2 * T * d * SIZE[case["dtype"]], flops=2 * T * K * numbers)


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("clip", "norm"):
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(v.double())) ** 2 for v in s["grads"]))
        at = torch.tensor(norm, dtype=torch.float64, device="cuda")
        if op == "norm":
            return at
        return dict(norm=at, out=[v.double() * min(1.0, case["max_norm"] / (norm + 1e-6)) for v in s["grads"]])
    grid = torch.tensor(sorted(set(E2M1)), dtype=torch.float64, device="cuda")
    if op == "quantize4":
        x = s["x"].double()
        if s["source"] is not None:
            x = x[torch.div(s["source"].long(), s["top_k"], rounding_mode="floor")]
        rows, D = x.shape
        if x.numel() > 1 << 28:                                        # some 2 GB a copy
            return None
        v = torch.cat([x, torch.zeros(rows, -D % BLOCK4, dtype=torch.float64, device="cuda")], 1).view(rows, -1, BLOCK4)
        s2 = torch.exp2(torch.ceil(torch.log2(v.abs().amax(2, keepdim=True).clamp_min(2.0 ** -100) / 6)))
        v = v / s2
        up = torch.searchsorted(grid, v.contiguous()).clamp(1, len(grid) - 1)      # grid[up - 1] < v <= grid[up]
        lo, hi = grid[up - 1], grid[up]
        even = (up - 7) % 2 == 0                                       # zero is number 7 of the grid, and even
        r = torch.where(v - lo < hi - v, lo, torch.where(v - lo > hi - v, hi, torch.where(even, hi, lo)))
        return (r * s2).view(rows, -1)[:, :D]

    def stands_for(q, scale, K):
        rows = q.view(torch.uint8).to(torch.int64)
        v = torch.empty(*rows.shape[:-1], 2 * rows.shape[-1], dtype=torch.float64, device="cuda")
        table = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
        v[..., 0::2], v[..., 1::2] = table[rows % 16], table[rows // 16]
        k = torch.arange(K, device="cuda") // BLOCK4
        return v[..., :K] * torch.exp2(scale.view(torch.uint8).double() - 127).index_select(-1, k)
    if op == "product4":
        a = stands_for(s["a"], s["a_scale"], s["K"])
        if not s["groups"]:
            return a @ stands_for(s["b"], s["b_scale"], s["K"]).T
        y = torch.empty(s["M"], s["N"], dtype=torch.float64, device=a.device)
        at = s["offsets"].tolist()
        for e in range(s["groups"]):
            y[at[e]:at[e + 1]] = a[at[e]:at[e + 1]] @ stands_for(s["b"][e], s["b_scale"][e], s["K"]).T
        return y

    # a layer: the choice as it is defined, token by token, then every assignment's two products
    x = s["x"].double()
    logits = s["logits"].double() if s["logits"] is not None else (x @ s["matrix"].double().T - s["shift"].double()) * TEMPERATURE
    p = torch.sigmoid(logits) if s["score"] == "sigmoid" else torch.softmax(logits, 1)
    G, E, T, K = s["groups"], s["E"], s["T"], s["top_k"]
    key = p + (0 if s["bias"] is None else s["bias"].double())
    if G > 1:
        in_group = key.view(T, G, E // G)
        rank = (-in_group.topk(2, dim=2).values.sum(2)).argsort(dim=1, stable=True).argsort(dim=1)
        key = torch.where((rank < (G + 1) // 2)[:, :, None], in_group, torch.full_like(in_group, -math.inf)).view(T, E)
    ids = (-key).argsort(dim=1, stable=True)[:, :K]
    w = p.gather(1, ids)
    w = 2.5 * w / w.sum(1, keepdim=True)

    def eight(v):                                                      # the rounding is defined in 32 bits
        v = v.float()
        out = torch.empty(v.shape, dtype=torch.float64, device=v.device)
        for b in range(0, v.shape[1], BLOCK):
            part = v[:, b:b + BLOCK]
            a = part.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
            out[:, b:b + BLOCK] = (part * (torch.full_like(a, 448.0) / a)).to(E4M3).double() * (a * (1.0 / 448.0)).double()
        return out

    def matrix(q, scale):
        r, k = torch.arange(q.shape[0], device=q.device) // BLOCK, torch.arange(q.shape[1], device=q.device) // BLOCK
        return q.double() * scale.double()[r][:, k]
    xq, y = eight(s["x"]), torch.zeros(T, s["d"], dtype=torch.float64, device="cuda")
    for e in ids.unique().tolist():
        t, j = (ids == e).nonzero(as_tuple=True)
        u = xq[t] @ matrix(s["w1"][e], s["w1_scale"][e]).T
        a, up = (u[:, :s["h"]], u[:, s["h"]:]) if s["gated"] else (u, 1.0)
        a = (torch.nn.functional.silu(a) if s["act"] == "silu" else a.clamp_min(0).square()) * up
        y.index_add_(0, t, w[t, j][:, None] * (eight(a) @ matrix(s["w2"][e], s["w2_scale"][e]).T))
    return y
