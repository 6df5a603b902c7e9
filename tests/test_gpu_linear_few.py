"""Dense layers of one row to some tens: up to eight, sixteen and 32 rows by a kernel of their own (wider layers of nine rows on by
tiles 32 rows wide), one row in the gradient, and in-place arguments at those sizes.

Against 64 bits, with the tolerances of test_gpu_encoder.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import BF16, F16, F32, activation, clean_status, close, gen, gs, normal, padded, rest, rounding  # noqa: E402, F401


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("fan_in,fan_out,name,dtype,keep", [
    (1, 1, "gelu", BF16, True), (31, 17, "silu", F16, False), (515, 300, "relu", BF16, True), (2049, 33, "none", F16, True),
    (264, 2368, "gelu", F16, False), (72, 2369, "silu", BF16, True), (130, 2500, "gelu", BF16, False), (8, 5003, "relu", F16, True)])
def test_few_rows(gs, rows, fan_in, fan_out, name, dtype, keep):  # noqa: F811
    g = gen(rows + fan_in + fan_out)
    x, w = normal(rows, fan_in, dtype, g, extra=1), normal(fan_out, fan_in, dtype, g, 1.5 * fan_in ** -0.5, extra=1)
    bias, r = torch.randn(fan_out, generator=g, device="cuda"), normal(rows, fan_out, dtype, g, extra=1)
    z, out = padded(rows, fan_out, dtype, extra=1) if keep else None, padded(rows, fan_out, dtype, extra=1)
    gs.linear(x, w, out, bias=bias, activation=name, residual=r, z=z)
    want_z = x.double() @ w.double().T + bias.double()
    off = (fan_in + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T) + 2.0 ** -23 * bias.double().abs() + 2.0 ** -24 * want_z.abs()
    y, _, special, _ = activation(want_z, name)
    want = y + r.double()
    close(out, want, rounding(want, dtype) + 1.2 * off + special + 2.0 ** -24 * want.abs())
    assert torch.isnan(rest(out)).all()
    if keep:
        close(z, want_z, rounding(want_z, dtype) + off)
        assert torch.isnan(rest(z)).all()
    over = padded(rows, fan_out, dtype).copy_(r)
    gs.linear(x, w, over, bias=bias, activation=name, residual=over)
    assert torch.equal(over, out)
    assert gs.device_status() == 0


@pytest.mark.parametrize("rows", [1, 2, 9, 40])
@pytest.mark.parametrize("fan_in,fan_out,name,dtype", [(1, 1, "gelu", F16), (33, 70, "silu", BF16), (520, 9, "relu", F16), (1000, 300, "none", BF16), (2500, 130, "gelu", BF16)])
def test_gradient_of_few_rows(gs, rows, fan_in, fan_out, name, dtype):  # noqa: F811
    g = gen(rows + fan_in)
    dz, w = normal(rows, fan_out, dtype, g, extra=1), normal(fan_out, fan_in, dtype, g, fan_out ** -0.5)
    x, below, a = normal(rows, fan_in, dtype, g), normal(rows, fan_in, dtype, g, 1.5), normal(rows, fan_in, dtype, g)
    dx, dz_below = padded(rows, fan_in, dtype).copy_(a), padded(rows, fan_in, dtype, extra=1)
    dw, db = padded(fan_out, fan_in, F32, extra=1), torch.full((fan_out,), float("nan"), device="cuda")
    gs.linear_backward(dz, x, w, dx=dx, dw=dw, db=db, around=dx, z_below=below, activation=name, dz_below=dz_below)      # (around in dx itself)
    want = dz.double() @ w.double() + a.double()
    off = (fan_out + 8) * 2.0 ** -23 * (dz.double().abs() @ w.double().abs()) + 2.0 ** -24 * want.abs()
    close(dx, want, rounding(want, dtype) + off)
    _, slope, _, special = activation(below.double(), name)
    full = want * slope
    close(dz_below, full, rounding(full, dtype) + off * slope.abs() + (special + 2.0 ** -24 * slope.abs()) * want.abs() + 2.0 ** -24 * full.abs())
    close(dw, dz.double().T @ x.double(), (rows + 8) * 2.0 ** -23 * (dz.double().abs().T @ x.double().abs()))
    close(db, dz.double().sum(0), (rows + 8) * 2.0 ** -23 * dz.double().abs().sum(0))
    assert torch.isnan(rest(dz_below)).all() and torch.isnan(rest(dw)).all()
    assert gs.device_status() == 0
