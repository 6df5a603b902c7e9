"""Activations and their slopes at infinities and NaN: kept sums of 16 bits may overflow to infinity, and one value has no say
in its neighbours (two are worked on at a time)."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import BF16, F16, activation, clean_status, close, gs, padded, rounding  # noqa: E402, F401

INF, NAN = math.inf, math.nan


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("name", ["relu", "gelu", "silu", "none"])
def test_slopes(gs, name, dtype):  # noqa: F811
    """Slopes of 1 at +infinity and 0 at -infinity (1 without an activation); a NaN's is NaN."""
    ends = [INF, 1.0, -INF, -2.0, NAN, 3.0, INF, -INF, NAN, NAN, 0.0, -0.0, -INF, 0.5, 7.0]
    z, d = padded(3, 15, dtype), padded(3, 15, dtype, fill=0.0)
    z.copy_(torch.tensor([ends, ends[::-1], ends[3:] + ends[:3]]))
    d += 2.0
    out = padded(3, 15, dtype)
    gs.activation_backward(d, z, name, out)
    odd = torch.isnan(z) & (name != "none")
    assert torch.equal(torch.isnan(out), odd)
    end = torch.isinf(z)
    want = torch.where(z > 0, 2.0, 0.0 if name != "none" else 2.0).to(dtype)
    assert torch.equal(out[end], want[end])
    rest = ~end & ~torch.isnan(z)
    _, slope, _, special = activation(z.double()[rest], name)
    close(out[rest], 2 * slope, rounding(2 * slope, dtype) + 2 * special + 2.0 ** -22 * slope.abs())


@pytest.mark.parametrize("rows", [5, 20, 100])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu", "none"])
def test_sums_at_the_ends(gs, name, rows):  # noqa: F811
    """A bias that is infinite or NaN: +infinity passes, NaN stays, ReLU of -infinity is 0; the other columns are as without."""
    x, w = torch.ones(rows, 16, dtype=BF16, device="cuda"), torch.zeros(33, 16, dtype=BF16, device="cuda")
    bias = torch.linspace(-3, 3, 33, device="cuda")
    plain, out = padded(rows, 33, BF16), padded(rows, 33, BF16)
    gs.linear(x, w, plain, bias=bias, activation=name)
    odd = bias.clone()
    odd[3::8], odd[4::8], odd[9::8] = INF, NAN, -INF
    gs.linear(x, w, out, bias=odd, activation=name)
    same = torch.isfinite(odd)
    assert torch.equal(out[:, same], plain[:, same])
    assert (out[:, odd == INF] == INF).all() and torch.isnan(out[:, torch.isnan(odd)]).all()
    if name in ("relu", "none"):
        assert (out[:, odd == -INF] == (0 if name == "relu" else -INF)).all()
