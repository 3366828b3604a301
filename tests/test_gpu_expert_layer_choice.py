"""The choice of experts in the whole layer's kernel is that of asgd_route, to the last bit; and forms of the call around it.

Both compute a score by the same operations in the same order (the softmax's sum over the lanes that asgd_route gives a token, the renormalising sum
over the lanes that hold its choices), so ids and weights are equal bit by bit, whatever hangs on the last one.  The logits here differ by some
steps of 2^-25 around a few levels: exponentials, their quotients and the sums with a bias then coincide or not by their last bits.
"""
import math

import pytest
import torch

import paper_1505_04956_b200 as pkg

from .test_gpu_expert_layer_serving import BF, F16, F32, _check, _gen, _matrices

pytestmark = pytest.mark.gpu


def _small_layer(g, E, d=16, h=16):
    """Experts that are all the same one."""
    w1, s1 = _matrices(g, 1, h, d)
    w2, s2 = _matrices(g, 1, d, h)
    many = lambda t: t.expand(E, *t.shape[1:]).contiguous() if t.dtype == F32 else t.view(torch.uint8).expand(E, *t.shape[1:]).contiguous().view(t.dtype)      # noqa: E731
    return many(w1), many(s1), many(w2), many(s2)


def _near(g, T, E, levels):
    """Logits around a few levels, 2^-25 and more apart."""
    level = torch.randint(0, levels, (T, E), generator=g, device="cuda").float() * 0.125
    return level + torch.randint(-6, 7, (T, E), generator=g, device="cuda").float() * 2.0 ** -25


@pytest.mark.parametrize("E, top_k, groups, kept, group_top", [
    (16, 2, 1, 1, 1), (33, 8, 1, 1, 1), (48, 6, 1, 1, 1), (64, 8, 1, 1, 1), (64, 9, 1, 1, 1), (64, 8, 8, 4, 2), (40, 4, 4, 2, 2), (48, 5, 16, 8, 2), (60, 7, 6, 6, 2),
    (12, 3, 3, 2, 1), (100, 8, 1, 1, 1), (256, 8, 8, 4, 2), (256, 32, 1, 1, 1), (300, 8, 1, 1, 1), (512, 16, 32, 8, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias, renormalise", [("zeros", True), ("some", False), ("none", True)])
def test_choices_that_hang_on_the_last_bit(E, top_k, groups, kept, group_top, score, bias, renormalise):
    g = _gen(E + top_k + groups)
    args = _small_layer(g, E)
    b = dict(none=None, zeros=torch.zeros(E, device="cuda"), some=torch.randint(0, 3, (E,), generator=g, device="cuda").float() * 2.0 ** -9)[bias]
    for T, levels in ((31, 3), (30, 1), (8, 2), (1, 1)):
        logits = _near(g, T, E, levels)
        x = torch.randn(T, 16, generator=g, device="cuda")
        kw = dict(score=score, bias=b, groups=groups, groups_kept=kept, group_top=group_top, renormalise=renormalise, scale=1.5)
        want_ids, want_weights = pkg.asgd_route(logits, top_k, plan=False, **kw)
        y, ids, weights = pkg.asgd_expert_layer(x, *args, top_k, logits=logits, choice=True, **kw)
        pkg.asgd_experts_sync()
        assert torch.equal(ids, want_ids)
        assert torch.equal(weights, want_weights)


@pytest.mark.parametrize("T, E, top_k, groups, kept", [(5, 300, 8, 1, 1), (7, 1000, 32, 1, 1), (16, 64, 4, 1, 1), (8, 96, 7, 6, 3), (40, 512, 16, 8, 8), (100, 33, 3, 11, 5), (2, 32, 32, 1, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", ["ties", "gone", "all equal"])
def test_weights_where_experts_are_unavailable(T, E, top_k, groups, kept, score, kind):
    g = _gen(T + E)
    logits = torch.randn(T, E, generator=g, device="cuda")
    if kind == "ties":
        logits = torch.round(logits * 2) / 2
    elif kind == "all equal":
        logits = torch.zeros(T, E, device="cuda")
    else:
        logits[torch.rand(T, E, generator=g, device="cuda") < 0.97] = -math.inf
        logits[T // 2] = -math.inf
    args = _small_layer(g, E)
    x = torch.randn(T, 16, generator=g, device="cuda")
    kw = dict(score=score, groups=groups, groups_kept=kept, group_top=1, scale=1.5)
    want_ids, want_weights = pkg.asgd_route(logits, top_k, plan=False, **kw)
    y, ids, weights = pkg.asgd_expert_layer(x, *args, top_k, logits=logits, choice=True, **kw)
    pkg.asgd_experts_sync()
    assert torch.equal(ids, want_ids) and torch.equal(weights, want_weights)
    assert bool((weights[ids < 0] == 0).all()) and bool((y[(ids < 0).all(1)] == 0).all())
    _check(x, *args, (y, ids, weights), "relu2", min_tight=False)


@pytest.mark.parametrize("T, E, top_k, groups, group_top, score, bias, renormalise, logits, act", [
    (8, 32, 4, 1, 1, "softmax", True, True, F32, "silu"), (40, 64, 8, 8, 2, "softmax", True, True, BF, "relu2"), (20, 96, 6, 6, 2, "softmax", False, False, F16, "silu"),
    (5, 128, 8, 1, 1, "softmax", True, False, BF, "relu2"), (33, 24, 3, 4, 2, "sigmoid", True, False, F32, "silu"), (3, 300, 8, 1, 1, "sigmoid", False, False, F16, "relu2"),
    (64, 16, 2, 1, 1, "softmax", False, False, BF, "silu")])
def test_forms_of_the_choice(T, E, top_k, groups, group_top, score, bias, renormalise, logits, act):
    g = _gen(3 * T + E)
    d, h = 272, 144
    x = torch.randn(T, d, generator=g, device="cuda").to(BF)
    w1, s1 = _matrices(g, E, 2 * h, d)
    w2, s2 = _matrices(g, E, d, h)
    lg = (torch.randn(T, E, generator=g, device="cuda") * 1.5).to(logits)
    kw = dict(score=score, bias=torch.randn(E, generator=g, device="cuda") * 0.1 if bias else None, groups=groups, groups_kept=(groups + 1) // 2,
              group_top=group_top, renormalise=renormalise, scale=2.0)
    want_ids, want_weights = pkg.asgd_route(lg, top_k, plan=False, **kw)
    got = pkg.asgd_expert_layer(x, w1, s1, w2, s2, top_k, logits=lg, activation=act, choice=True, **kw)
    pkg.asgd_experts_sync()
    assert torch.equal(got[1], want_ids) and torch.equal(got[2], want_weights)
    _check(x, w1, s1, w2, s2, got, act)


@pytest.mark.parametrize("T, router", [(1, F32), (9, BF), (50, F16)])
def test_a_router_without_shift(T, router):
    g = _gen(T)
    E, top_k, d, h = 24, 3, 300, 100
    x = torch.randn(T, d, generator=g, device="cuda")
    w1, s1 = _matrices(g, E, h, d)
    w2, s2 = _matrices(g, E, d, h)
    matrix = (torch.randn(E, d, generator=g, device="cuda") / d ** 0.5).to(router)
    got = pkg.asgd_expert_layer(x, w1, s1, w2, s2, top_k, router=matrix, temperature=0.5, choice=True)
    zero = pkg.asgd_expert_layer(x, w1, s1, w2, s2, top_k, router=matrix, shift=torch.zeros(E, device="cuda"), temperature=0.5, choice=True)
    pkg.asgd_experts_sync()
    assert all(torch.equal(a, b) for a, b in zip(got, zero))
    _check(x, w1, s1, w2, s2, got, "relu2")
    want_ids, _ = pkg.asgd_route(((x.double() @ matrix.double().t()) * 0.5).float(), top_k, plan=False)
    assert int((got[1] != want_ids).any(1).sum()) <= 1                             # a token whose choice hangs on the last bits


@pytest.mark.parametrize("T, E, top_k", [(128, 16, 2), (100, 64, 8), (70, 200, 1), (31, 3, 3), (16, 300, 2)])
def test_one_expert_has_all_tokens(T, E, top_k):
    """Several chunks of one expert, where the mean load is a small one."""
    g = _gen(T * E)
    d, h = 256, 200
    x = torch.randn(T, d, generator=g, device="cuda").to(BF)
    w1, s1 = _matrices(g, E, 2 * h, d)
    w2, s2 = _matrices(g, E, d, h)
    logits = torch.randn(T, E, generator=g, device="cuda")
    logits[:, E // 2] = 9.0
    got = pkg.asgd_expert_layer(x, w1, s1, w2, s2, top_k, logits=logits, activation="silu", choice=True)
    pkg.asgd_experts_sync()
    assert bool((got[1][:, 0] == E // 2).all())
    _check(x, w1, s1, w2, s2, got, "silu")


@pytest.mark.parametrize("E, top_k, d, h, gated, logits", [(2, 1, 65536, 16, True, True), (2, 2, 16, 65536, False, False), (1, 1, 4104, 32768, True, False)])
def test_the_widest_layers(E, top_k, d, h, gated, logits):
    g = _gen(d + h)
    x = torch.randn(3, d, generator=g, device="cuda")
    w1, s1 = _matrices(g, E, h * (2 if gated else 1), d)
    w2, s2 = _matrices(g, E, d, h)
    kw = dict(logits=torch.randn(3, E, generator=g, device="cuda")) if logits else dict(router=torch.randn(E, d, generator=g, device="cuda") / d ** 0.5)
    got = pkg.asgd_expert_layer(x, w1, s1, w2, s2, top_k, activation="silu", choice=True, **kw)
    pkg.asgd_experts_sync()
    _check(x, w1, s1, w2, s2, got, "silu", min_tight=False)


NAN_KW = [dict(score="softmax"), dict(score="sigmoid"), dict(score="sigmoid", groups=4, groups_kept=2, group_top=2)]


@pytest.mark.parametrize("kw", NAN_KW, ids=["softmax", "sigmoid", "groups"])
@pytest.mark.parametrize("T", [6, 40])
@pytest.mark.parametrize("dtype, router, d", [(F32, F32, 256), (BF, F32, 333), (F16, BF, 1030)])
def test_a_nan_and_an_infinity_reach_their_tokens_results_through_a_router(kw, T, dtype, router, d):
    """A token that is not finite has no logit to choose by; its result is not one of a token without experts."""
    g = _gen(T + d)
    E, top_k, h = 8, 2, 128
    x = torch.randn(T, d, generator=g, device="cuda").to(dtype)
    args = (*_matrices(g, E, 2 * h, d), *_matrices(g, E, d, h), top_k)
    matrix = torch.randn(E, d, generator=g, device="cuda") / d ** 0.5
    matrix[:, 7] = -matrix[:, 7].abs() - 0.01                                      # an infinity there makes every logit -inf
    kw = dict(kw, router=matrix.to(router), activation="silu", shift=torch.randn(E, generator=g, device="cuda") * 0.1)
    want = pkg.asgd_expert_layer(x, *args, **kw)
    bad = x.clone()
    bad[1, 0], bad[2, d - 1], bad[3, 7], bad[4, 9] = math.nan, math.nan, math.inf, math.inf
    got, ids, weights = pkg.asgd_expert_layer(bad, *args, choice=True, **kw)
    pkg.asgd_experts_sync()
    assert bool((ids[1:4] == -1).all()) and bool((weights[1:4] == 0).all())
    assert bool(torch.isnan(got[1:4]).all())
    assert not bool(torch.isfinite(got[4]).all())
    keep = [t for t in range(T) if t not in (1, 2, 3, 4)]
    assert torch.equal(got[keep], want[keep])


def test_a_finite_token_whose_logits_overflow_is_not_passed_over():
    g = _gen(12)
    E, top_k, d, h = 4, 2, 256, 128
    x = torch.randn(3, d, generator=g, device="cuda")
    x[1, :128], x[1, 128:] = 3e38, -3e38                                           # sums of infinities of both signs
    args = (*_matrices(g, E, 2 * h, d), *_matrices(g, E, d, h), top_k)
    got, ids, _ = pkg.asgd_expert_layer(x, *args, router=torch.full((E, d), 1e3, device="cuda"), choice=True)
    pkg.asgd_experts_sync()
    assert bool((ids[1] == -1).all()) and bool(torch.isnan(got[1]).all())


@pytest.mark.parametrize("dtype", [F32, BF])
def test_finite_tokens_without_an_expert_are_zeros(dtype):
    g = _gen(11)
    E, top_k, d, h = 4, 2, 260, 128
    x = torch.randn(5, d, generator=g, device="cuda").to(dtype)
    args = (*_matrices(g, E, 2 * h, d), *_matrices(g, E, d, h), top_k)
    matrix = torch.randn(E, d, generator=g, device="cuda")
    away = torch.full((E,), math.inf, device="cuda")                               # every expert's shift takes it out
    assert bool((pkg.asgd_expert_layer(x, *args, router=matrix, shift=away) == 0).all())
    logits = torch.full((5, E), -math.inf, device="cuda")                          # given logits take the token out, whatever it holds
    x[2] = math.nan
    assert bool((pkg.asgd_expert_layer(x, *args, logits=logits) == 0).all())
    pkg.asgd_experts_sync()


def test_a_factor_that_changes_in_place_counts_as_it_is_at_the_call():
    g = _gen(5)
    args = _small_layer(g, 8)
    x, logits = torch.randn(4, 16, generator=g, device="cuda"), torch.randn(4, 8, generator=g, device="cuda")
    scale = torch.tensor(1.0)
    for value in (1.0, 2.5):
        scale.fill_(value)
        _, _, weights = pkg.asgd_expert_layer(x, *args, 2, logits=logits, scale=scale, choice=True)
        assert torch.equal(weights, pkg.asgd_expert_layer(x, *args, 2, logits=logits, scale=value, choice=True)[2])
        assert torch.equal(pkg.asgd_route(logits, 2, scale=scale, plan=False)[1], pkg.asgd_route(logits, 2, scale=value, plan=False)[1])
    pkg.asgd_experts_sync()
