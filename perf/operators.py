"""The operators of a layer of experts, as cases that can be timed and compared: routing, 8-bit block-scaled
operands and their products, and the combination of the experts' rows.

With `own` false every operator is computed in its plain form (elementary torch operations in 32 bits, rounded once
at the end); with `own` true by the calls a user makes of the framework.
"""
import math

import torch

own = False

FMAX = {"e4m3": 448.0, "e5m2": 57344.0}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # a serving step of eight sequences: scores by sigmoid, a balance bias, groups of experts; latency is all
        dict(name="route, 8 tokens", op="route", T=8, E=256, top_k=8, score="sigmoid", groups=8, kept=4, group_top=2, dtype="bf16", align=1),
        # a training batch's tokens routed by softmax, rows of every expert padded to whole blocks of 128
        dict(name="route, 16384 tokens", op="route", T=16384, E=128, top_k=8, score="softmax", groups=1, kept=1, group_top=1, dtype="f32", align=128),
        # the gradient of the same choice on a long batch
        dict(name="route gradient", op="route_grad", T=32768, E=64, top_k=2, score="softmax", dtype="bf16"),
        # tokens gathered into their experts' order on the way to 8 bits (input of the experts' first product)
        dict(name="quantize into experts", op="quantize", T=8192, D=4096, top_k=4, form="rows", dtype="bf16", fmt="e4m3"),
        # an output gradient of odd sizes laid out for both of its products (input and weight gradient) at once
        dict(name="quantize both ways", op="quantize", T=4001, D=2056, top_k=0, form="both", dtype="f32", fmt="e5m2"),
        # one serving step of five sequences through a dense layer: the weights' bytes
        dict(name="product, 5 rows", op="product", M=5, N=4096, K=4096, groups=0, fmt="e4m3", out="bf16"),
        # a prompt or training batch through a large dense layer: the tensor pipe's rate
        dict(name="product, 8192 rows", op="product", M=8192, N=8192, K=8192, groups=0, fmt="e4m3", out="bf16"),
        # a serving step through 64 experts, a handful of rows each and some with none: every expert's weights once
        dict(name="experts, 256 rows", op="product", M=256, N=2048, K=2048, groups=64, fmt="e4m3", out="bf16"),
        # a batch through 32 experts of uneven load and odd sizes
        dict(name="experts, 16384 rows", op="product", M=16384, N=2744, K=2064, groups=32, fmt="e4m3", out="bf16"),
        # the experts' weight gradients: the sum runs over each expert's own rows
        dict(name="experts' weight gradient", op="weight_grad", R=16384, N=2048, K=2048, groups=16, fmt="e4m3", out="f32"),
        # the experts' rows back into token order, weighted
        dict(name="combine, 8192 tokens", op="combine", T=8192, D=4096, top_k=4, dtype="bf16"),
        # its gradient: to the rows and to the routing weights
        dict(name="combine gradient", op="combine_grad", T=5003, D=2560, top_k=6, dtype="bf16"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    v = max(step * -(-lo // step), min(v, hi // step * step))
    return v if v != 3 << 10 else v + step


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "quantize", "quantize", "product", "product", "product", "product",
                     "weight_grad", "combine", "combine_grad"])
    if op == "route":
        score = rng.choice(["softmax", "sigmoid"])
        groups = rng.choice([1, 1, 4, 8])
        per = _log(rng, 4, 256 // groups)
        kept = rng.randint(1, groups)
        return dict(op=op, T=_log(rng, 1, 65536), E=groups * per, top_k=rng.randint(1, min(8, kept * per)), score=score,
                    groups=groups, kept=kept, group_top=2 if score == "sigmoid" and groups > 1 else 1,
                    dtype=rng.choice(["f32", "bf16", "f16"]), align=rng.choice([1, 128]))
    if op == "route_grad":
        E = _log(rng, 4, 256)
        return dict(op=op, T=_log(rng, 1, 65536), E=E, top_k=rng.randint(1, min(8, E)), score=rng.choice(["softmax", "sigmoid"]),
                    dtype=rng.choice(["f32", "bf16", "f16"]))
    if op == "quantize":
        top_k = rng.choice([0, 0, 2, 4, 8])
        return dict(op=op, T=_log(rng, 1, 8192 if top_k < 8 else 4096), D=_log(rng, 128, 8192, rng.choice([1, 8, 128])), top_k=top_k,
                    form=rng.choice(["rows", "both"] if top_k else ["rows", "both", "blocks"]),
                    dtype=rng.choice(["f32", "bf16", "f16"]), fmt=rng.choice(["e4m3", "e5m2"]))
    if op == "product":
        groups = rng.choice([0, 0, 8, 32, 64])
        return dict(op=op, M=_log(rng, 1, 16384 if groups else 8192), N=_log(rng, 256, 4096, 8), K=_log(rng, 256, 4096, rng.choice([16, 128])),
                    groups=groups, fmt=rng.choice(["e4m3", "e4m3", "e5m2"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if op == "weight_grad":
        groups = rng.choice([1, 8, 16, 32])
        return dict(op=op, R=_log(rng, 1024, 32768, 128), N=_log(rng, 256, 2048, 8), K=_log(rng, 256, 2048, 8), groups=groups,
                    fmt=rng.choice(["e4m3", "e5m2"]), out=rng.choice(["f32", "bf16"]))
    return dict(op=op, T=_log(rng, 1, 8192), D=_log(rng, 256, 4096, rng.choice([1, 8])), top_k=rng.randint(1, 8), dtype=rng.choice(["f32", "bf16", "f16"]))


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _loads(rng_cpu, groups, rows, unit):
    """Rows per group: a skewed multinomial (popular and unpopular experts, some with nothing), whole units."""
    p = torch.rand(groups, generator=rng_cpu).pow(2) + 0.01
    n = torch.multinomial(p, rows // unit, replacement=True, generator=rng_cpu)
    return torch.bincount(n, minlength=groups) * unit


def _operand(g, shape, fmt, block_rows):
    """An 8-bit operand [..., rows, K] and its scales [..., rows / block_rows, K / 128] as a quantiser leaves them: values
    of unit variance with every 61st column ten times as large."""
    K = shape[-1]
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., ::61] *= 10
    kb = _ceil(K, BLOCK)
    pad = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, -shape[-2] % block_rows))
    v = pad.reshape(*pad.shape[:-2], pad.shape[-2] // block_rows, block_rows, kb, BLOCK)
    amax = v.abs().amax(dim=(-3, -1)).clamp_min(2.0 ** -100)
    inv = torch.full_like(amax, FMAX[fmt]) / amax
    q = (v * inv.unsqueeze(-1).unsqueeze(-3)).reshape(pad.shape)[..., :shape[-2], :K].to(FP8[fmt])
    scale = amax * (1.0 / FMAX[fmt])
    ld = _ceil(K, 16) * 16
    if ld != K:                                                  # rows start at multiples of 16 bytes
        store = torch.zeros(*shape[:-1], ld, dtype=torch.uint8, device="cuda")
        store[..., :K] = q.view(torch.uint8)
        q = store[..., :K].view(FP8[fmt])
    else:
        q = q.contiguous()
    if block_rows == 1:
        scale = scale.transpose(-1, -2).contiguous().transpose(-1, -2)      # block after block, as the quantiser lays them out
    return q, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.Generator().manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op in ("route", "route_grad"):
        # hidden states against router rows, some experts more popular than others
        pop = torch.randn(case["E"], generator=g, device="cuda") * 0.5
        s["logits"] = (torch.randn(case["T"], case["E"], generator=g, device="cuda") * 1.5 + pop).to(DTYPE[case["dtype"]])
        if op == "route":
            s["bias"] = torch.randn(case["E"], generator=g, device="cuda") * 0.1 if case["score"] == "sigmoid" else None
        else:
            s["ids"] = torch.topk(s["logits"].float(), case["top_k"], dim=1).indices.to(torch.int32)
            s["dweights"] = torch.randn(case["T"], case["top_k"], generator=g, device="cuda")
    elif op == "quantize":
        x = torch.randn(case["T"], case["D"], generator=g, device="cuda")
        x *= torch.exp(torch.randn(case["T"], 1, generator=g, device="cuda"))
        x[:, ::67] *= 10
        s["x"] = x.to(DTYPE[case["dtype"]])
        s["source"] = torch.randperm(case["T"] * case["top_k"], generator=g, device="cuda").to(torch.int32) if case["top_k"] else None
    elif op == "product":
        s["a"], s["a_scale"] = _operand(g, (case["M"], case["K"]), case["fmt"], 1)
        w = (case["groups"], case["N"], case["K"]) if case["groups"] else (case["N"], case["K"])
        s["b"], s["b_scale"] = _operand(g, w, "e4m3", BLOCK)
        s["offsets"] = None
        if case["groups"]:
            n = _loads(c, case["groups"], case["M"], 1)
            s["most"] = int(n.max())
            s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).cuda()
    elif op == "weight_grad":
        s["a"], s["a_scale"] = _operand(g, (case["N"], case["R"]), case["fmt"], 1)
        s["b"], s["b_scale"] = _operand(g, (case["K"], case["R"]), "e4m3", 1)
        n = _loads(c, case["groups"], case["R"], BLOCK)
        s["most"] = int(n.max())
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).cuda()
    else:
        T, K, D, dt = case["T"], case["top_k"], case["D"], DTYPE[case["dtype"]]
        s["z"] = torch.randn(T * K, D, generator=g, device="cuda").to(dt)
        perm = torch.randperm(T * K, generator=g, device="cuda")
        s["source"] = perm.to(torch.int32)
        rows = torch.empty_like(perm)
        rows[perm] = torch.arange(T * K, device="cuda")
        s["rows"] = rows.reshape(T, K).to(torch.int32)
        w = torch.rand(T, K, generator=g, device="cuda") + 0.05
        s["weights"] = w / w.sum(1, keepdim=True)
        if op == "combine_grad":
            s["dy"] = torch.randn(T, D, generator=g, device="cuda").to(dt)
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else PLAIN[s["op"]](s)


def _own(s):
    import paper_1505_04956_b200 as pkg
    op = s["op"]
    if op == "route":
        ids, weights, offsets, rows, source = pkg.asgd_route(
            s["logits"], s["top_k"], bias=s["bias"], score=s["score"], groups=s["groups"], groups_kept=s["kept"],
            group_top=s["group_top"], renormalise=True, scale=2.5, align=s["align"])
        return dict(ids=ids, weights=weights, offsets=offsets, rows=rows, source=source)
    if op == "route_grad":
        return pkg.asgd_route_grad(s["logits"], s["ids"], s["dweights"], score=s["score"], renormalise=True, scale=2.5)
    if op == "quantize":
        return pkg.asgd_quantize(s["x"], form=s["form"], dtype=FP8[s["fmt"]], source=s["source"], per_token=max(1, s["top_k"]))
    if op == "product":
        return pkg.asgd_product(s["a"], s["a_scale"], s["b"], s["b_scale"], offsets=s["offsets"], out_dtype=DTYPE[s["out"]])
    if op == "weight_grad":
        return pkg.asgd_product_inner(s["a"], s["a_scale"], s["b"], s["b_scale"], s["offsets"], out_dtype=DTYPE[s["out"]])
    if op == "combine":
        return pkg.asgd_combine(s["z"], s["rows"], s["weights"])
    return pkg.asgd_combine_grad(s["dy"], s["z"], s["rows"], s["weights"], s["source"])


# ---- plain forms, 32 bits ----

def _scores(x, score):
    if score == "sigmoid":
        return torch.reciprocal(torch.exp(-x) + 1.0)
    e = torch.exp(x - x.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(s):
    x = s["logits"].float()
    T, E, K, G = s["T"], s["E"], s["top_k"], s["groups"]
    p = _scores(x, s["score"])
    key = x if s["bias"] is None and s["group_top"] == 1 else p if s["bias"] is None else p + s["bias"]
    if G > 1:
        best = key.reshape(T, G, E // G).sort(dim=2, descending=True).values
        of_group = best[..., 0] + best[..., 1] if s["group_top"] == 2 and E // G > 1 else best[..., 0]
        kept = of_group.sort(dim=1, descending=True, stable=True).indices[:, :s["kept"]]
        out = torch.ones(T, G, dtype=torch.bool, device=x.device).scatter(1, kept, False)
        key = key.masked_fill(out.repeat_interleave(E // G, dim=1), -math.inf)
    ids = key.sort(dim=1, descending=True, stable=True).indices[:, :K]
    w = p.gather(1, ids)
    w = 2.5 * w / (w.sum(1, keepdim=True) + 1e-20)
    # the plan: assignments grouped by expert in ascending order, every expert's rows from a multiple of `align`
    flat, align = ids.reshape(-1), s["align"]
    n = torch.zeros(E, dtype=torch.int64, device=x.device).scatter_add(0, flat, torch.ones_like(flat))
    zero = torch.zeros(1, dtype=torch.int64, device=x.device)
    first = torch.cat([zero, n.cumsum(0)])
    offsets = torch.cat([zero, ((n + align - 1) // align * align).cumsum(0)])
    by, order = flat.sort(stable=True)
    place = offsets[by] + torch.arange(T * K, device=x.device) - first[by]
    rows = torch.empty_like(flat).scatter(0, order, place)
    source = torch.full((T * K + E * (align - 1),), -1, dtype=torch.int64, device=x.device).scatter(0, place, order)
    return dict(ids=ids.int(), weights=w, offsets=offsets.int(), rows=rows.reshape(T, K).int(), source=source.int())


def _plain_route_grad(s):
    x = s["logits"].float()
    ids, dw = s["ids"].long(), s["dweights"]
    p = _scores(x, s["score"])
    c = p.gather(1, ids)
    total = c.sum(1, keepdim=True) + 1e-20
    ds = 2.5 * (dw - (dw * c).sum(1, keepdim=True) / total) / total
    if s["score"] == "sigmoid":
        dx = torch.zeros_like(x).scatter(1, ids, ds * c * (1 - c))
    else:
        dx = p * (torch.zeros_like(x).scatter(1, ids, ds) - (ds * c).sum(1, keepdim=True))
    return dx.to(s["logits"].dtype)


def _plain_blocks(x, bm, bn, fmt):
    """8-bit values of x and the scales of its bm x bn blocks."""
    M, N = x.shape
    pad = torch.nn.functional.pad(x, (0, -N % bn, 0, -M % bm))
    v = pad.reshape(pad.shape[0] // bm, bm, pad.shape[1] // bn, bn)
    amax = v.abs().amax(dim=(1, 3)).clamp_min(2.0 ** -100)
    inv = torch.full_like(amax, FMAX[fmt]) / amax
    q = (v * inv[:, None, :, None]).reshape(pad.shape)[:M, :N].to(FP8[fmt])
    return q, amax * (1.0 / FMAX[fmt])


def _plain_quantize(s):
    x = s["x"].float()
    if s["source"] is not None:
        x = x[s["source"].long() // s["top_k"]]
    if s["form"] == "blocks":
        return _plain_blocks(x, BLOCK, BLOCK, s["fmt"])
    rows = _plain_blocks(x, 1, BLOCK, s["fmt"])
    return rows if s["form"] == "rows" else rows + _plain_blocks(x.t().contiguous(), 1, BLOCK, s["fmt"])


def _values(q, scale):
    """8-bit operand times its scales in 32 bits."""
    rows, K = q.shape[-2:]
    sc = scale.repeat_interleave(BLOCK, dim=-2)[..., :rows, :] if scale.shape[-2] != rows else scale
    return q.float() * sc.repeat_interleave(BLOCK, dim=-1)[..., :K]


def _plain_product(s):
    a, b = _values(s["a"], s["a_scale"]), _values(s["b"], s["b_scale"])
    dt = DTYPE[s["out"]]
    if not s["groups"]:
        return (a @ b.t()).to(dt)
    M, most = s["M"], s["most"]
    at = s["offsets"][:-1, None].long() + torch.arange(most, device=a.device)
    at = torch.where(at < s["offsets"][1:, None], at, M)
    a = torch.cat([a, torch.zeros_like(a[:1])])
    y = torch.empty(M + 1, s["N"], device=a.device)
    y[at.reshape(-1)] = torch.bmm(a[at], b.transpose(1, 2)).reshape(-1, s["N"])
    return y[:M].to(dt)


def _plain_weight_grad(s):
    a, b = _values(s["a"], s["a_scale"]), _values(s["b"], s["b_scale"])
    R, most = s["R"], s["most"]
    at = s["offsets"][:-1, None].long() + torch.arange(most, device=a.device)
    at = torch.where(at < s["offsets"][1:, None], at, R)
    a = torch.cat([a, torch.zeros_like(a[:, :1])], 1)[:, at].transpose(0, 1)
    b = torch.cat([b, torch.zeros_like(b[:, :1])], 1)[:, at].permute(1, 2, 0)
    return torch.bmm(a, b).to(DTYPE[s["out"]])


def _plain_combine(s):
    z = s["z"].float()[s["rows"].long()]
    return (z * s["weights"][..., None]).sum(1).to(s["z"].dtype)


def _plain_combine_grad(s):
    dy, src = s["dy"].float(), s["source"].long()
    dz = dy[src // s["top_k"]] * s["weights"].reshape(-1)[src][:, None]
    dw = (s["z"].float()[s["rows"].long()] * dy[:, None]).sum(2)
    return dz.to(s["z"].dtype), dw


PLAIN = dict(route=_plain_route, route_grad=_plain_route_grad, quantize=_plain_quantize, product=_plain_product,
             weight_grad=_plain_weight_grad, combine=_plain_combine, combine_grad=_plain_combine_grad)


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("route", "route_grad"):
        T, E, K = case["T"], case["E"], case["top_k"]
        if op == "route":
            plan = 4 * (E + 1) + 4 * T * K + 4 * (T * K + E * (case["align"] - 1))
            return dict(bytes=T * E * SIZE[case["dtype"]] + 8 * T * K + plan, flops=T * E * 4)
        return dict(bytes=2 * T * E * SIZE[case["dtype"]] + 8 * T * K, flops=T * E * 6)
    if op == "quantize":
        T, D = case["T"], case["D"]
        R = T * max(1, case["top_k"])
        forms = 2 if case["form"] == "both" else 1
        scales = _ceil(R, BLOCK) * _ceil(D, BLOCK) if case["form"] == "blocks" else R * _ceil(D, BLOCK) + (D * _ceil(R, BLOCK) if forms == 2 else 0)
        return dict(bytes=T * D * SIZE[case["dtype"]] + forms * R * D + 4 * scales + (4 * R if case["top_k"] else 0), flops=2 * R * D * forms)
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        # weights of the experts that have rows, on average over the loads that _loads() draws
        G = case["groups"]
        used = sum(1 - math.exp(-M * (((i + 0.5) / 64) ** 2 + 0.01) / (G * (1 / 3 + 0.01))) for i in range(64)) / 64 * G if G else 1
        return dict(bytes=M * K + 4 * M * _ceil(K, BLOCK) + round(used * (N * K + 4 * _ceil(N, BLOCK) * _ceil(K, BLOCK))) + M * N * SIZE[case["out"]],
                    flops=2 * M * N * K)
    if op == "weight_grad":
        R, N, K = case["R"], case["N"], case["K"]
        return dict(bytes=(N + K) * (R + 4 * _ceil(R, BLOCK)) + case["groups"] * N * K * SIZE[case["out"]], flops=2 * R * N * K)
    T, D, K = case["T"], case["D"], case["top_k"]
    if op == "combine":
        return dict(bytes=T * (K + 1) * D * SIZE[case["dtype"]] + 8 * T * K, flops=2 * T * K * D)
    return dict(bytes=T * (2 * K + 1) * D * SIZE[case["dtype"]] + 16 * T * K, flops=3 * T * K * D)


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        x = s["logits"].double()
        p = torch.sigmoid(x) if s["score"] == "sigmoid" else torch.softmax(x, 1)
        key = x if s["bias"] is None and s["group_top"] == 1 else p + (0 if s["bias"] is None else s["bias"].double())
        G, E = s["groups"], s["E"]
        if G > 1:
            in_group = key.view(-1, G, E // G)
            of_group = in_group.topk(min(s["group_top"], E // G), dim=2).values.sum(2)
            rank = (-of_group).argsort(dim=1, stable=True).argsort(dim=1)
            key = torch.where((rank < s["kept"])[:, :, None], in_group, torch.full_like(in_group, -math.inf)).view(-1, E)
        ids = (-key).argsort(dim=1, stable=True)[:, :s["top_k"]]
        w = p.gather(1, ids)
        return dict(ids=None, weights=2.5 * w / w.sum(1, keepdim=True), offsets=None, rows=None, source=None)
    if op == "route_grad":
        x = s["logits"].double().requires_grad_()
        p = torch.sigmoid(x) if s["score"] == "sigmoid" else torch.softmax(x, 1)
        c = p.gather(1, s["ids"].long())
        (2.5 * c / (c.sum(1, keepdim=True) + 1e-20)).backward(s["dweights"].double())
        return x.grad
    if op == "quantize":
        x = s["x"].double()
        if s["source"] is not None:
            x = x[torch.div(s["source"].long(), s["top_k"], rounding_mode="floor")]

        def largest(t, bm, bn):
            M, N = t.shape
            m = torch.nn.functional.pad(t.abs(), (0, -N % bn, 0, -M % bm)).unflatten(1, (-1, bn)).amax(2)
            return m.unflatten(0, (-1, bm)).amax(1) / FMAX[s["fmt"]]
        # the scales; of the 8-bit values the rounding is the definition, and what they stand for follows from it
        if s["form"] == "blocks":
            return None, largest(x, BLOCK, BLOCK)
        rows = (None, largest(x, 1, BLOCK))
        return rows if s["form"] == "rows" else rows + (None, largest(x.t(), 1, BLOCK))

    def stands_for(q, scale):
        rows, K = q.shape[-2:]
        r = torch.arange(rows, device=q.device) // (1 if scale.shape[-2] == rows else BLOCK)
        k = torch.arange(K, device=q.device) // BLOCK
        return q.double() * scale.double().index_select(-2, r).index_select(-1, k)
    if op == "product":
        a = stands_for(s["a"], s["a_scale"])
        if not s["groups"]:
            return a @ stands_for(s["b"], s["b_scale"]).T
        y = torch.empty(s["M"], s["N"], dtype=torch.float64, device=a.device)
        at = s["offsets"].tolist()
        for e in range(s["groups"]):
            y[at[e]:at[e + 1]] = a[at[e]:at[e + 1]] @ stands_for(s["b"][e], s["b_scale"][e]).T
        return y
    if op == "weight_grad":
        a, b, at = stands_for(s["a"], s["a_scale"]), stands_for(s["b"], s["b_scale"]), s["offsets"].tolist()
        return torch.stack([a[:, at[e]:at[e + 1]] @ b[:, at[e]:at[e + 1]].T for e in range(s["groups"])])
    w = s["weights"].double()
    if op == "combine":
        y = torch.zeros(s["T"], s["D"], dtype=torch.float64, device=w.device)
        for j in range(s["top_k"]):
            y += w[:, j:j + 1] * s["z"][s["rows"][:, j].long()].double()
        return y
    dz = torch.zeros(s["T"] * s["top_k"], s["D"], dtype=torch.float64, device=w.device)
    dw = torch.zeros_like(w)
    for j in range(s["top_k"]):
        r = s["rows"][:, j].long()
        dz[r] = w[:, j:j + 1] * s["dy"].double()
        dw[:, j] = (s["dy"].double() * s["z"][r].double()).sum(1)
    return dz, dw
