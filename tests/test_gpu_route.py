"""Routing of tokens to experts and its gradient against plain implementations in 64 bits."""
import math

import pytest
import torch

from experts_util import order_of, route64
from operators_util import DTYPE, close, rand

pytestmark = pytest.mark.gpu
# Weights: the exponential of a difference below 32 that is rounded once (2^-19) or, without renorm, of one below 64 (2^-18), the exponential's two units in
# the last place, the logarithm of the sigmoid, a sum of up to 32 and a division: less than 2^-17 of the value.
WEIGHT = 2.0 ** -17


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def check(sp, logits, k, **how):
    weights, experts = sp.route(logits, k, **how)
    want_w, want_e = route64(logits, k, **how)
    assert experts.dtype == torch.int32 and torch.equal(experts, want_e)
    close(weights, want_w, "f32", WEIGHT * want_w.abs())
    return weights, experts


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 8), (3, 31, 2), (33, 64, 6), (130, 65, 1), (70, 128, 8), (37, 256, 8), (9, 257, 32), (5, 1024, 16)])
def test_choice(sp, t, score, renorm, T, E, k):
    logits = rand((T, E), t, T + E, 1.5, pad=3)
    check(sp, logits, k, score=score, renorm=renorm, scale=2.5)
    check(sp, logits, k, score=score, renorm=renorm, bias=rand((E,), "f32", 7, 0.2))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 3, 6), (256, 8, 4, 8), (60, 5, 1, 12), (32, 32, 4, 4), (1024, 32, 7, 20), (6, 2, 2, 6)])
def test_groups(sp, score, group_score, bias, E, groups, top_groups, k):
    for t in ("f32", "bf16"):
        logits = rand((45, E), t, E + groups, 1.5)
        check(sp, logits, k, score=score, groups=groups, top_groups=top_groups, group_score=group_score, bias=rand((E,), "f32", 3, 0.1) if bias else None)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [None, "zeros", "equal", "near"])
@pytest.mark.parametrize("groups", [1, 4])
def test_ties(sp, score, bias, groups):
    """Logits of few values: the lower index first; and sums that FP32 cannot tell apart but 64 bits can."""
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randint(-2, 3, (64, 64), generator=g, device="cuda").to(torch.bfloat16)
    b = {None: None, "zeros": torch.zeros(64, device="cuda"), "equal": torch.full((64,), 0.3, device="cuda"),
         "near": 0.25 + torch.arange(64, device="cuda") * 2.0 ** -25}[bias]
    check(sp, logits, 8, score=score, bias=b, groups=groups, top_groups=max(1, groups // 2), group_score="top2" if groups > 1 else "max")


def test_close_scores_are_told_apart_in_64_bits(sp):
    """f32 logits one unit in the last place apart, under a bias that swallows the difference in FP32."""
    base = torch.full((16, 40), 0.7, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = (base.view(torch.int32) + torch.randint(0, 4, base.shape, generator=g, device="cuda", dtype=torch.int32)).view(torch.float32)
    for score in ("softmax", "sigmoid"):
        check(sp, logits, 6, score=score, bias=torch.full((40,), 0.5, device="cuda"))
        check(sp, logits, 6, score=score, bias=torch.full((40,), -8.0, device="cuda"), groups=4, top_groups=2, group_score="top2")


@pytest.mark.parametrize("E", [64, 128, 256, 40])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_pairs_and_triples_of_close_scores(sp, score, E):
    """Steps of 0.05 with one, two or three logits each, some equal and some a unit in the last place apart, in any places of the row."""
    g = torch.Generator(device="cuda").manual_seed(E)
    T = 400
    level = (torch.arange(E, device="cuda") // 2).float() * 0.05
    level[2::7] = level[1::7][:len(level[2::7])]
    units = torch.randint(0, 3, (T, E), generator=g, device="cuda", dtype=torch.int32)
    logits = ((level + 0.0173).expand(T, E).contiguous().view(torch.int32) + units).view(torch.float32)
    logits = torch.gather(logits, 1, torch.rand((T, E), generator=g, device="cuda").argsort(1))
    for bias in (0.5, -3.0):
        b = torch.full((E,), bias, device="cuda")
        check(sp, logits, 8, score=score, bias=b)
        check(sp, logits, 3, score=score, bias=b, groups=4, top_groups=2, group_score="top2")
        check(sp, logits, 3, score=score, groups=4, top_groups=3, group_score="top2")


def test_masked_experts_and_tokens(sp):
    for t in ("bf16", "f32"):
        logits = rand((40, 48), t, 5, 1.5)
        g = torch.Generator(device="cuda").manual_seed(3)
        logits[torch.rand((40, 48), generator=g, device="cuda") < 0.85] = -math.inf   # (tokens with fewer than six)
        logits[7] = -math.inf
        for how in ({}, {"score": "sigmoid"}, {"renorm": False}, {"bias": rand((48,), "f32", 1, 0.1)}, {"groups": 4, "top_groups": 2},
                    {"groups": 4, "top_groups": 2, "group_score": "top2", "score": "sigmoid", "bias": rand((48,), "f32", 1, 0.1)}):
            weights, experts = check(sp, logits, 6, **how)
            assert bool((experts[7] == -1).all()) and bool((weights[7] == 0).all())
    bias = rand((48,), "f32", 1, 0.1)
    bias[::2] = -math.inf
    check(sp, rand((40, 48), "f32", 6), 6, score="sigmoid", bias=bias)


def test_what_is_not_finite(sp):
    logits = rand((6, 32), "f32", 8)
    logits[1, 4], logits[2, 9], logits[3, 2] = math.nan, math.inf, torch.finfo(torch.float32).min
    logits[4] = torch.finfo(torch.float32).min       # (a mask by the lowest value: all equal)
    logits[5] = -200.0                               # sigmoids that are all 0 in FP32
    clean = logits.clone()
    clean[1, 4] = -math.inf
    weights, experts = sp.route(logits, 4)
    assert torch.equal(experts, route64(clean, 4)[1]) and bool(weights[1].isnan().all()) and bool(weights[2].isnan().all())
    rows = [0, 3, 4, 5]
    close(weights[rows], route64(clean, 4)[0][rows], "f32", WEIGHT)
    weights, experts = sp.route(logits, 4, score="sigmoid")
    want = route64(clean, 4, score="sigmoid")
    assert torch.equal(experts, want[1]) and bool(weights[1].isnan().all())
    close(weights[[0, 2, 3, 5]], want[0][[0, 2, 3, 5]], "f32", WEIGHT)


def test_probabilities_over_a_wide_range(sp):
    logits = rand((64, 96), "f32", 9, 30.0)
    check(sp, logits, 8, score="softmax")
    check(sp, logits, 8, score="sigmoid")
    check(sp, logits, 8, score="sigmoid", renorm=False)


def gradient64(dweights, logits, experts, score, renorm, scale):
    """Differentiated by autograd, in 64 bits."""
    l = logits.double().clone().requires_grad_()
    live = (experts >= 0) & (experts < logits.shape[1])
    at = torch.where(live, experts, torch.zeros_like(experts)).long()
    z = torch.log_softmax(l, 1) if score == "softmax" else torch.nn.functional.logsigmoid(l)
    picked = torch.gather(z, 1, at).masked_fill(~live, -math.inf)
    some = live.any(1)
    w = torch.softmax(picked[some], 1) if renorm else torch.exp(picked[some])
    grad, = torch.autograd.grad((w * scale * dweights[some].double()).masked_fill(~live[some], 0).sum(), l)
    return torch.nan_to_num(grad)


# Gradient: scores off by 2^-18 (as above), differences of the g of up to `size` = the largest |g| of the token.
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 8, 3), (33, 64, 6), (9, 257, 32), (3, 1024, 8), (260, 128, 4)])
def test_gradient(sp, t, score, renorm, T, E, k):
    logits = rand((T, E), t, T + E, 1.5, pad=1)
    g = rand((T, k), "f32", 4)
    _, experts = sp.route(logits, k, score=score)
    if T > 4:
        experts[1], experts[2, 0], experts[3, k - 1] = -1, -1, E + 5
    got = sp.route_backward(g, logits, experts, score=score, renorm=renorm, scale=2.5)
    want = gradient64(g, logits, experts, score, renorm, 2.5)
    assert got.dtype == DTYPE[t]
    close(got, want, t, 2.0 ** -15 * 2.5 * g.double().abs().amax(1, keepdim=True))


def test_gradient_against_differences(sp):
    """The weights change by what the gradient says, with steps that stay far from another choice."""
    logits, g = rand((16, 24), "f32", 11), rand((16, 4), "f32", 12)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            _, experts = sp.route(logits, 4, score=score, renorm=renorm)
            d = sp.route_backward(g, logits, experts, score=score, renorm=renorm).double()
            step = rand((16, 24), "f32", 13).double()
            z = lambda l: torch.log_softmax(l, 1) if score == "softmax" else torch.nn.functional.logsigmoid(l)  # noqa: E731
            f = lambda l: ((torch.softmax(v, 1) if renorm else torch.exp(v)) * g.double()).sum(1) if (v := torch.gather(z(l), 1, experts.long())) is not None else None  # noqa: E731
            h = 1e-4
            slope = (f(logits.double() + h * step) - f(logits.double() - h * step)) / (2 * h)
            # a central difference is off by h^2 times the third derivative (below 64 for steps of a few units); the gradient as above
            assert bool(((d * step).sum(1) - slope).abs().max() <= 64 * h * h * 100 + 2.0 ** -15 * 24 * 4)


def test_gradient_in_place_and_twice_the_same_expert(sp):
    logits, g = rand((7, 40), "f16", 1), rand((7, 3), "f32", 2)
    experts = torch.tensor([[1, 1, 5]] * 7, dtype=torch.int32, device="cuda")
    for renorm in (True, False):
        want = gradient64(g, logits, experts, "softmax", renorm, 1.0)
        there = logits.clone()
        got = sp.route_backward(g, there, experts, renorm=renorm, out=there)
        assert got is there
        close(got, want, "f16", 2.0 ** -15 * g.double().abs().amax(1, keepdim=True))


@pytest.mark.parametrize("E", [1, 5, 64, 1000, 1024])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 8), (7, 3), (300, 2), (2049, 4), (40000, 8)])
@pytest.mark.parametrize("align", [1, 16, 24])
def test_order(sp, E, T, k, align):
    g = torch.Generator(device="cuda").manual_seed(E + T)
    experts = (torch.randn((T, k), generator=g, device="cuda").abs() * E / 2).to(torch.int32)   # some are not below E
    experts[torch.rand((T, k), generator=g, device="cuda") < 0.1] = -1
    order = sp.expert_order(experts, E, align=align)
    for got, want in zip(order, order_of(experts, E, align)):
        assert got.dtype == torch.int32 and torch.equal(got.cpu(), want)


def test_order_of_nothing(sp):
    order = sp.expert_order(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 6)
    assert order.offsets.tolist() == [0] * 7 and order.position.shape == (0, 4) and order.source.shape == (0,)
    order = sp.expert_order(torch.full((5, 2), -1, dtype=torch.int32, device="cuda"), 6, align=16)
    assert order.offsets.tolist() == [0] * 7 and bool((order.position == -1).all()) and bool((order.source == -1).all())
    weights, experts = sp.route(torch.empty((0, 8), device="cuda"), 2)
    assert weights.shape == experts.shape == (0, 2)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [32, 64, 96, 128, 160, 192, 256])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (2, 1), (4, 3), (8, 4)])
def test_chunks_of_experts_and_single_ones_agree(sp, t, score, E, groups, top_groups):
    """Rows of whole vectors go through other kernels than rows between boundaries; masks, infinities, NaN and ties among them."""
    g = torch.Generator(device="cuda").manual_seed(E + groups)
    wide = torch.randn((203, E + 1), generator=g, device="cuda").mul_(1.5).to(DTYPE[t])
    wide[torch.rand(wide.shape, generator=g, device="cuda") < 0.1] = -math.inf
    wide[3], wide[4, 5], wide[5, 7], wide[6] = -math.inf, math.nan, math.inf, 0.5
    wide[7:9, :E // 2] = 0.25
    whole = wide[:, 1:].contiguous()
    for bias in (None, rand((E,), "f32", 3, 0.2), torch.zeros(E, device="cuda"), torch.where(torch.arange(E, device="cuda") % 3 == 0, -math.inf, 0.125)):
        for by in ("max", "top2"):
            for renorm in (True, False):
                for k in (1, 3, 8):
                    if k > top_groups * (E // groups):
                        continue
                    how = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_score=by, renorm=renorm)
                    a, b = sp.route(whole, k, **how), sp.route(wide[:, 1:], k, **how)
                    assert torch.equal(a[1], b[1]), (bias is None, by, renorm, k)
                    close(a[0], b[0].double(), "f32", WEIGHT * b[0].double().abs())
    check(sp, whole[10:60], min(8, top_groups * (E // groups)), score=score, bias=rand((E,), "f32", 3, 0.2), groups=groups, top_groups=top_groups, group_score="top2")
