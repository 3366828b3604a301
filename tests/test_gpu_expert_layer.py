"""The layer of experts behind learnt centres: its gradients against autograd in fp32, and a short training run."""
import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import expert_layer

pytestmark = pytest.mark.gpu


def test_gradients_are_those_of_the_layer_in_fp32():
    # Rounding to E4M3 changes a number by up to 2^-4 of itself, 3.6 % in the mean square; to E5M2 twice that.  A product of
    # two rounded operands is off by the root of the sum of squares; the longest chain here (w1: tokens, first matrix,
    # squared hidden values, second matrix, two gradients in E5M2) has 2 x 3.6 (the square doubles the first product's 5 %),
    # 3.6, 3.6 and 2 x 7.2 %, together below 20 %.
    tokens, d, experts, hidden = 1500, 128, 4, 256
    X, target = expert_layer.make_task(tokens, d, experts, seed=3)
    layer = expert_layer.make_layer(X, experts, hidden, seed=3)
    y, c = layer.forward(X)
    dy = torch.randn(tokens, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    got = layer.gradients(X, dy, c)
    pkg.asgd_experts_sync()

    x = X.clone().requires_grad_()
    router, w1, w2 = (t.clone().requires_grad_() for t in (layer.router, layer.w1, layer.w2))
    s = torch.sigmoid((x @ router.t() - layer.shift) * layer.temperature).gather(1, c["ids"].long())
    w = s / s.sum(1, keepdim=True)
    want_y = torch.zeros_like(x)
    for j in range(layer.top_k):
        for e in range(experts):
            m = c["ids"][:, j] == e
            want_y[m] = want_y[m] + w[m, j:j + 1] * (torch.relu(x[m] @ w1[e].t()).square() @ w2[e].t())
    want = torch.autograd.grad((want_y * dy).sum(), (router, w1, w2, x))
    rel = lambda a, b: float((a - b).norm() / b.norm())                   # noqa: E731
    assert rel(y, want_y.detach()) < 0.2
    for name, a, b in zip(("router", "w1", "w2", "x"), got, want):
        assert rel(a, b) < 0.2, name


def test_a_short_training_run_learns():
    first, last = expert_layer.main(tokens=2048, d=128, experts=4, hidden=256, steps=31)
    assert last < 0.7 * first
