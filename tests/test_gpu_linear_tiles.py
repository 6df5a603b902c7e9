"""Dense layers where a pair of thread blocks works on several tiles, one after the other: the two sets of sums alternate, what
the epilogue reads of a tile is fetched during the tile before, and tiles without a feature or a row for a warp come
between those that have some.

Against 64 bits, with the tolerances of test_gpu_encoder.py: (n + 8) 2^-23 times the sum of the magnitudes of a dot
product's n terms, what the activations' special functions may be off by, one rounding a sum and the output's."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import ACTS, BF16, F16, activation, clean_status, close, gen, gs, normal, padded, rest, rounding  # noqa: E402, F401

# rows, features of the result, length of the contraction.  Tiles are 256 features by 32 to 256 rows, dealt out to 74 pairs in turn;
# the width is the one whose rounds take the shortest.
SIZES = [
    (30011, 600, 130),       # 256 rows wide, 354 tiles: full and partial ones (88 of 256 features) in turn, four or five a pair
    (20000, 1160, 72),       # 256, 395 tiles: the last of five holds 136 features, so that a CTA of the pair has eight of them
    (25003, 603, 72),        # 256, 294 tiles: the last piece of eight features holds three
    (20005, 333, 40),        # 256, 158 tiles: 77 of 256 features, the last piece five
    (6200, 600, 264),        # 128, 147 tiles: two a pair; the last row tile has 56 rows
    (6150, 530, 40),         # 128, 147 tiles, the last row tile six rows: nothing for the warps of its second half
    (40, 40000, 64),         # 64, 157 tiles
    (20, 39000, 72),         # 32, 153 tiles
]


def spread(rows, cols, dtype, g, scale):
    """Every value its own (a mix-up of rows or columns anywhere shows)."""
    return normal(rows, cols, dtype, g, scale, extra=1)


@pytest.mark.parametrize("rows,features,depth", SIZES)
@pytest.mark.parametrize("name,dtype,residual,keep", [("gelu", BF16, True, True), ("none", F16, True, False), ("relu", BF16, False, True), ("silu", F16, True, False)])
def test_forward(gs, rows, features, depth, name, dtype, residual, keep):  # noqa: F811
    g = gen(rows + features + depth)
    x, w, bias = spread(rows, depth, dtype, g, 1.0), spread(features, depth, dtype, g, 1.5 * depth ** -0.5), torch.randn(features, generator=g, device="cuda")
    r = spread(rows, features, dtype, g, 1.0) if residual else None
    z, out = padded(rows, features, dtype, extra=1) if keep else None, padded(rows, features, dtype, extra=2)
    gs.linear(x, w, out, bias=bias, activation=name, residual=r, z=z)
    want_z = x.double() @ w.double().T
    off = (depth + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T) + 2.0 ** -23 * bias.double().abs()
    want_z += bias.double()
    off += 2.0 ** -24 * want_z.abs()
    y, _, special, _ = activation(want_z, name)
    want = y if r is None else y + r.double()
    close(out, want, rounding(want, dtype) + 1.2 * off + special + 2.0 ** -24 * want.abs())
    assert torch.isnan(rest(out)).all()
    if keep:
        close(z, want_z, rounding(want_z, dtype) + off)
        assert torch.isnan(rest(z)).all()
    for _ in range(3):                           # the same every time, in place of the residual too, and no wait ran out
        again = padded(rows, features, dtype)
        if residual:
            again.copy_(r)
        gs.linear(x, w, again, bias=bias, activation=name, residual=again if residual else None)
        assert torch.equal(again, out)
    assert gs.device_status() == 0


@pytest.mark.parametrize("rows,features,depth", SIZES)
@pytest.mark.parametrize("name,dtype,around,both", [("gelu", BF16, True, True), ("relu", F16, True, False), ("silu", BF16, False, True), ("none", F16, True, True)])
def test_gradient_of_the_rows(gs, rows, features, depth, name, dtype, around, both):  # noqa: F811
    g = gen(rows + features + depth + 1)
    dz, w = spread(rows, depth, dtype, g, 1.0), spread(depth, features, dtype, g, depth ** -0.5)
    below = spread(rows, features, dtype, g, 1.5)
    a = spread(rows, features, dtype, g, 1.0) if around else None
    x = padded(rows, features, dtype)            # (read for the gradient of the weights alone: left as NaN)
    dx, dz_below = padded(rows, features, dtype, extra=1) if both else None, padded(rows, features, dtype, extra=2)
    gs.linear_backward(dz, x, w, dx=dx, around=a, z_below=below, activation=name, dz_below=dz_below)
    want = dz.double() @ w.double()
    off = (depth + 8) * 2.0 ** -23 * (dz.double().abs() @ w.double().abs())
    if around:
        want += a.double()
    off += 2.0 ** -24 * want.abs()
    if both:
        close(dx, want, rounding(want, dtype) + off)
        assert torch.isnan(rest(dx)).all()
    _, slope, _, special = activation(below.double(), name)
    full = want * slope
    close(dz_below, full, rounding(full, dtype) + off * slope.abs() + (special + 2.0 ** -24 * slope.abs()) * want.abs() + 2.0 ** -24 * full.abs())
    assert torch.isnan(rest(dz_below)).all()
    for _ in range(3):                           # the same every time, `around` in dx itself too
        over, again = padded(rows, features, dtype), padded(rows, features, dtype)
        if around:
            over.copy_(a)
        gs.linear_backward(dz, x, w, dx=over if both else None, around=(over if both else a) if around else None, z_below=below, activation=name, dz_below=again)
        assert torch.equal(again, dz_below) and (not both or torch.equal(over, dx))
    assert gs.device_status() == 0


@pytest.mark.parametrize("fan_in", [4096, 65536])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_long_sums_of_one_sign(gs, fan_in, dtype):  # noqa: F811
    """The documented drift, 6e-9 of a sum's value a term (held here to 2^-27 a term), and the output's rounding; the order of the
    terms inside an instruction is off by 2^-20 at most."""
    g = gen(fan_in)
    x = (torch.rand(500, fan_in, generator=g, device="cuda") + 0.5).to(dtype)
    w = ((torch.rand(72, fan_in, generator=g, device="cuda") + 0.5) / fan_in).to(dtype)
    out, dx = padded(500, 72, dtype), padded(500, 72, dtype)
    gs.linear(x, w, out)
    gs.linear_backward(x, padded(500, 72, dtype), w.T.contiguous(), dx=dx)
    want = x.double() @ w.double().T
    room = rounding(want, dtype) + (2.0 ** -27 * fan_in + 2.0 ** -20) * want
    close(out, want, room)
    close(dx, want, room)
