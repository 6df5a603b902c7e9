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
