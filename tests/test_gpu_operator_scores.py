"""Scores, weights and their gradients where floats run out of range or of digits: large scales, rows with
nothing left, scores far below the best one.

u is the unit roundoff of a float, 2^-24.  A score passes through the subtraction of the row's largest logit d = x - top
(|d| u of the exponential, nothing where the difference is exact), an exponential (2 units), a sum of up to 512
terms in 32 lanes (32 u) and two divisions: 2^-18 holds it beside |d| u.  Below 2^-126 a float has fewer digits:
2^-149 absolute."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operators import BF16, F16, F32, UNIT, clean_status, close, gen, gs, route  # noqa: E402, F401

LEAST = 2.0 ** -149


def router_of(experts, top_k, **more):
    from paper_2605_16867_b200 import ExpertRouter
    return ExpertRouter(experts, top_k, **more)


@pytest.mark.parametrize("experts", [9, 33])                 # a thread and a warp per row
@pytest.mark.parametrize("n", [300, 5000])                   # one launch, several
@pytest.mark.parametrize("scale", [3.5e18, -1e30, 3.4e38])
def test_weights_of_any_scale(gs, experts, n, scale):  # noqa: F811
    x = torch.randn(n, experts, generator=gen(1), device="cuda")
    x[::3] = -math.inf                                       # nothing left
    x[1::3, 2:] = -math.inf                                  # fewer than top_k
    for bias in (None, torch.zeros(experts, device="cuda")):
        unit = route(gs, x, router_of(experts, 3), bias)
        expert, weight, *_ = route(gs, x, router_of(experts, 3, scale=scale), bias)
        assert torch.equal(expert, unit[0])
        assert (weight[expert < 0] == 0).all() and (expert[::3] == -1).all()
        close(weight, unit[1].double() * scale, 2.0 ** -22 * abs(scale) * unit[1].double())
    assert gs.device_status() == 0


def exact_scores(x, score):
    x = x.double()
    return torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)


@pytest.mark.parametrize("experts", [9, 16, 32, 40, 200])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_scores_far_below_the_best(gs, experts, score, dtype):  # noqa: F811
    """Every score of rows whose logits spread over a hundred and more, in steps that all types hold exactly."""
    k = min(16, experts)
    for n in (60, 4000):
        g = gen(experts + n)
        x = (torch.randint(-240, 200, (n, experts), generator=g, device="cuda").float() / 4).to(dtype)
        expert, weight, *_ = route(gs, x, router_of(experts, k, score=score, renormalise=False))
        s = exact_scores(x, score)
        want = s.gather(1, expert.long())
        close(weight, want, 2.0 ** -18 * want + 2 * LEAST)
        if experts <= 16 and score == "softmax":             # all of them were chosen, the largest first (sigmoids meet at one)
            held = s.float()
            order = torch.sort(torch.where(held >= 4 * LEAST, held, 0.0), dim=1, descending=True, stable=True)[1]
            clear = (torch.sort(held, dim=1, descending=True)[0][:, :k] >= 4 * LEAST)
            assert torch.equal(expert[clear].long(), order[:, :k][clear])
        # weights of a dense choice add up to one
        _, weight, *_ = route(gs, x, router_of(experts, k, score=score))
        total = want.sum(1, keepdim=True) + 1e-20
        close(weight, want / total, 2.0 ** -18 * want / total + 4 * LEAST / total.clamp_max(1.0))
    assert gs.device_status() == 0


@pytest.mark.parametrize("experts,groups", [(9, 1), (40, 1), (64, 8)])
def test_choice_below_the_least_normal_score(gs, experts, groups):  # noqa: F811
    """One expert takes all but e^-88 and less; the next places go by what is left, not by the index."""
    for n in (50, 4000):
        x = torch.full((n, experts), -200.0, device="cuda")
        x[:, 5], x[:, 3], x[:, 6], x[:, 1] = 0.0, -95.0, -90.0, -99.0
        router = router_of(experts, 4, n_groups=groups, top_groups=groups)
        expert, weight, *_ = route(gs, x, router)
        assert expert.unique(dim=0).tolist() == [[5, 6, 3, 1]]
        want = torch.tensor([0.0, -90.0, -95.0, -99.0], device="cuda").double().exp().expand(n, 4)
        close(weight, want, 2.0 ** -18 * want + 4 * LEAST)
    assert gs.device_status() == 0


@pytest.mark.parametrize("experts", [9, 31, 33, 100, 256])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_gradient_of_saturated_sigmoids(gs, experts, renormalise, dtype):  # noqa: F811
    """dx = dq s (1 - s): held to 2^-17 of the sum of dq's terms' magnitudes times s (1 - s), then rounded once."""
    k = min(8, experts)
    router = router_of(experts, k, score="sigmoid", renormalise=renormalise)
    for n in (1, 500):
        g = gen(experts)
        x = ((torch.rand(n, experts, generator=g, device="cuda") * 2 - 1) * 25).to(dtype)
        x[:, 0], x[:, -1] = 18.0, -30.0
        expert = route(gs, x, router)[0].long()
        dw = torch.randn(n, k, generator=g, device="cuda")
        out = torch.empty_like(x)
        gs.expert_route_backward(x, router, expert.int(), dw, out)
        s, rest = torch.sigmoid(x.double()), torch.sigmoid(-x.double())
        q, dwd = s.gather(1, expert), dw.double()
        t = q.sum(1, keepdim=True) + 1e-20
        dq = (dwd - (dwd * q).sum(1, keepdim=True) / t) / t if renormalise else dwd
        room = (dwd.abs() + (dwd.abs() * q).sum(1, keepdim=True) / t) / t if renormalise else dwd.abs()
        slope = (s * rest).gather(1, expert)
        want, mag = (torch.zeros_like(s).scatter_add_(1, expert, v * slope) for v in (dq, room))
        assert (want.abs().amax(1) > 0).all()
        close(out, want, 2.0 ** -17 * mag + UNIT[dtype] * want.abs() + (2.0 ** -25 if dtype is F16 else 1e-37))
    assert gs.device_status() == 0
