"""A layer of experts behind learnt centres, trained end to end (python -m paper_1505_04956_b200.expert_layer).

The workers of the K-Means loop learn k centres of the tokens; a centre's row becomes the router's row of one expert, so
that a token's logits rank the centres by distance.  The experts are two matrices each with a squared rectifier between
them.  A step runs every operator of the layer: routing and its gradient, tokens rounded to 8 bits on their way into the
experts' order, the experts' products and both of their gradients, and the sum back into token order with its gradient.
The task is the regression of a seeded function that differs from cluster to cluster.
"""
from __future__ import annotations

import dataclasses

import torch

from . import inputs
from .binding import Asgd, make_config
from .experts import (asgd_combine, asgd_combine_grad, asgd_experts_sync, asgd_product, asgd_product_inner, asgd_quantize, asgd_route,
                      asgd_route_grad)
from .gradients import asgd_clip_grads
from .serving import asgd_expert_layer

ALIGN = 128                     # grouped rows per block of the weight gradients' sums
E5M2 = torch.float8_e5m2        # gradients have the wider range


def learn_centres(X, k, seed=0):
    """k centres [k, d] of the rows of X by the worker loop, one pass over the samples."""
    W = 4
    wl = inputs.WORKLOADS["mid"].scaled(N=X.shape[0], d=X.shape[1], k=k, W=W, b=min(128, X.shape[0] // W), seed=seed)
    cfg = make_config(N=wl.N, d=wl.d, k=k, W=W, b=wl.b, eps=1.0, comm_interval=4, fanout=1, seed=seed)
    ctx = Asgd(cfg, X, inputs.initial_centres(wl, X))
    ctx.step(4 * wl.B)
    ctx.sync()
    centres = ctx.get_state(-1)
    ctx.destroy()
    return centres


def eight_bits(w):
    """An expert's matrices [E, n, k] in 8 bits, as they are and transposed, with the scales of their 128 x 128 blocks."""
    parts = [asgd_quantize(m, form="blocks both") for m in w]
    q, s, qt = (torch.stack([p[i] for p in parts]) for i in range(3))
    return (q, s), (qt, s.transpose(1, 2).contiguous())


@dataclasses.dataclass
class Layer:
    """fp32 master weights.  router [E, d], shift [E] (the centres' half squared norms), w1 [E, h, d], w2 [E, d, h], and the
    balance bias, which takes part in the choice alone."""
    router: torch.Tensor
    shift: torch.Tensor
    w1: torch.Tensor
    w2: torch.Tensor
    bias: torch.Tensor
    top_k: int = 2
    temperature: float = 0.05

    def logits(self, x):
        return (x @ self.router.t() - self.shift) * self.temperature

    def forward(self, x):
        """y [T, d] fp32, and what the gradients need."""
        logits = self.logits(x)
        ids, weights, offsets, rows, source = asgd_route(logits, self.top_k, score="sigmoid", bias=self.bias, align=ALIGN)
        w1, w1t = eight_bits(self.w1)
        w2, w2t = eight_bits(self.w2)
        xq, xs, xqt, xst = asgd_quantize(x, form="both", source=source, per_token=self.top_k)
        u = asgd_product(xq, xs, *w1, offsets=offsets)
        r = torch.relu(u.float())
        hq, hs, hqt, hst = asgd_quantize(r * r, form="both")
        z = asgd_product(hq, hs, *w2, offsets=offsets, out_dtype=torch.float32)
        y = asgd_combine(z, rows, weights)
        return y, dict(logits=logits, ids=ids, weights=weights, offsets=offsets, rows=rows, source=source, r=r, z=z,
                       xt=(xqt, xst), ht=(hqt, hst), w1t=w1t, w2t=w2t)

    def eight_bits(self):
        """The experts' matrices as serve() takes them: for steps that change nothing they are made once."""
        return tuple(eight_bits(w)[0] for w in (self.w1, self.w2))

    def serve(self, x, weights=None):
        """y of the few tokens of a serving step (128 at most, 1024 choices of experts), of x's type; `weights` as eight_bits() gives them.
        With them it is one call of the library; without, every matrix is rounded to 8 bits first, in every call.  Numbers between the two products are
        fp32 here, while forward() rounds the first one's results to bf16, so the two differ by some per cent of y's norm."""
        (w1, s1), (w2, s2) = self.eight_bits() if weights is None else weights
        return asgd_expert_layer(x, w1, s1, w2, s2, self.top_k, router=self.router, shift=self.shift, temperature=self.temperature,
                                 activation="relu2", score="sigmoid", bias=self.bias)

    def gradients(self, x, dy, c):
        """Gradients of router, w1 and w2 and of the layer's input, from dy [T, d] fp32."""
        dz, dweights = asgd_combine_grad(dy, c["z"], c["rows"], c["weights"], c["source"])
        dzq, dzs, dzqt, dzst = asgd_quantize(dz, form="both", dtype=E5M2)
        dw2 = asgd_product_inner(dzqt, dzst, *c["ht"], c["offsets"])
        dh = asgd_product(dzq, dzs, *c["w2t"], offsets=c["offsets"], out_dtype=torch.float32)
        duq, dus, duqt, dust = asgd_quantize(2.0 * dh * c["r"], form="both", dtype=E5M2)
        dw1 = asgd_product_inner(duqt, dust, *c["xt"], c["offsets"])
        dxg = asgd_product(duq, dus, *c["w1t"], offsets=c["offsets"], out_dtype=torch.float32)
        dlogits = asgd_route_grad(c["logits"], c["ids"], dweights, score="sigmoid")
        dx = asgd_combine(dxg, c["rows"]) + self.temperature * dlogits @ self.router
        return self.temperature * dlogits.t() @ x, dw1, dw2, dx

    def step(self, x, target, rate, balance=0.002, max_norm=None):
        """One step of gradient descent on the mean squared error, its gradients clipped to `max_norm` together where that is given;
        returns the error (a tensor) and the experts' loads."""
        y, c = self.forward(x)
        diff = y - target
        drouter, dw1, dw2, _ = self.gradients(x, diff * (2.0 / diff.numel()), c)
        if max_norm is not None:
            asgd_clip_grads((drouter, dw1, dw2), max_norm)
        self.router -= 0.05 * rate * drouter                    # the centres are learnt already
        self.w1 -= rate * dw1
        self.w2 -= rate * dw2
        loads = torch.bincount(c["ids"].reshape(-1) + 1, minlength=self.bias.numel() + 1)[1:]
        self.bias += balance * torch.sign(loads.float().mean() - loads)
        return diff.square().mean(), loads


def make_layer(X, experts, hidden, top_k=2, seed=0):
    g = torch.Generator(device=X.device).manual_seed(seed)
    d = X.shape[1]
    centres = learn_centres(X, experts, seed)
    draw = lambda *shape: torch.randn(*shape, generator=g, device=X.device)      # noqa: E731
    return Layer(centres, 0.5 * centres.square().sum(1), draw(experts, hidden, d) / d ** 0.5, draw(experts, d, hidden) * (0.5 / hidden ** 0.5),
                 torch.zeros(experts, device=X.device), top_k)


def make_task(tokens, d, clusters, seed=0):
    """Tokens from a mixture, and a target that is another linear map in every cluster."""
    wl = inputs.WORKLOADS["mid"].scaled(N=tokens, d=d, k=clusters, seed=seed, means="normal:1", sigma=0.3)
    X, comp = inputs.make_samples(wl, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    maps = torch.randn(clusters, d, d, generator=g, device="cuda") / d ** 0.5
    of = torch.cdist(X, inputs.mixture_parameters(wl, "cuda")[0]).argmin(1)
    target = torch.empty_like(X)
    for e in range(clusters):
        target[of == e] = X[of == e] @ maps[e]
    return X, target


def main(tokens=8192, d=256, experts=8, hidden=512, steps=60, rate=1.0, max_norm=None):
    X, target = make_task(tokens, d, experts)
    layer = make_layer(X, experts, hidden)
    first = last = None
    for i in range(steps):
        loss, loads = layer.step(X, target, rate, max_norm=max_norm)
        if i % 10 == 0 or i == steps - 1:
            last = float(loss)
            first = last if first is None else first
            print("step %3d  mean squared error %.4f  loads %s" % (i, last, loads.tolist()), flush=True)
    asgd_experts_sync()
    return first, last


if __name__ == "__main__":
    main()
