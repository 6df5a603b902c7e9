"""The experts' products where a pair of thread blocks works on several tiles, one after the other: the ring of
operand stages, the two sets of sums and the experts' rows carry over from tile to tile.

Tolerances as in test_gpu_operators.py: (n + 8) * 2^-23 times the sum of the magnitudes of a dot product's n
terms, then one rounding to the output's type."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operators import BF16, F16, UNIT, clean_status, close, gen, gs, layout, normal, of_rows, padded, rest, segments  # noqa: E402, F401


def uneven(experts, rows, g):
    """Rows of every expert, adding up to `rows`: some far above the mean, some none, some one."""
    share = torch.rand(experts, generator=g, device="cuda").pow(2) + 0.05
    counts = (share / share.sum() * (rows - experts)).long()
    counts[1::7], counts[2::11] = 0, 1
    counts[0] += rows - counts.sum()
    return counts.tolist()


# experts, rows, in, out: the average expert's rows choose the tile's width; at least three tiles for each of 74 pairs
# in both directions
TILES = [
    (300, 4100, 400, 1100),                     # 32 wide
    (150, 6000, 300, 700),                      # 64
    (90, 9001, 600, 520),                       # 128
    (9, 20003, 520, 1030),                      # 256
]


def tiles_id(c):
    return f"{c[0]}e-{c[1]}r-{c[2]}-{c[3]}"


def inputs(case, gather, dtype):
    experts, rows, i, o = case
    g = gen(rows)
    counts = uneven(experts, rows, g)
    offsets, rows, row_token = layout(counts, g, rows // 2 if gather else None)
    x = normal(rows // 2 if gather else rows, i, dtype, g, extra=1)
    w = padded(experts * o, i, dtype)
    w.copy_(torch.randn(experts * o, i, generator=g, device="cuda") * i ** -0.5)
    return g, offsets, rows, row_token, x, w.unflatten(0, (experts, o)), torch.randn(experts, o, generator=g, device="cuda")


@pytest.mark.parametrize("case", TILES, ids=tiles_id)
@pytest.mark.parametrize("gather", [False, True], ids=["in-order", "gathered"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_rows_over_several_tiles_of_a_pair(gs, case, gather, dtype):  # noqa: F811
    experts, _, i, o = case
    g, offsets, rows, row_token, x, w, bias = inputs(case, gather, dtype)
    dz = normal(rows, o, dtype, g)
    out, dx = padded(rows, o, dtype, extra=1), padded(rows, i, dtype, extra=1)
    gs.expert_linear(x, w, offsets, out, bias=bias, row_token=row_token, relu=True)
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx, row_token=row_token, relu_input=True)
    xs, zs = of_rows(x, row_token).double(), dz.double()
    for e, r in segments(offsets):
        we = w[e].double()
        want = (xs[r] @ we.T + bias[e].double()).clamp_min(0)
        mag = xs[r].abs() @ we.abs().T + bias[e].double().abs()
        close(out[r], want, (i + 8) * 2.0 ** -23 * mag + UNIT[dtype] * want.abs() + 2.0 ** -25)
        want = torch.where(xs[r] > 0, zs[r] @ we, 0.0)
        close(dx[r], want, (o + 8) * 2.0 ** -23 * (zs[r].abs() @ we.abs()) + UNIT[dtype] * want.abs() + 2.0 ** -25)
    assert torch.isnan(rest(out)).all() and torch.isnan(rest(dx)).all()
    for _ in range(5):                          # the same every time, and no wait ran out
        again, back = padded(rows, o, dtype), padded(rows, i, dtype)
        gs.expert_linear(x, w, offsets, again, bias=bias, row_token=row_token, relu=True)
        gs.expert_linear_backward(dz, x, w, offsets, dx=back, row_token=row_token, relu_input=True)
        assert torch.equal(again, out) and torch.equal(back, dx)
    assert gs.device_status() == 0


def cut_inputs(case, gather, dtype):
    """Experts with more rows than one piece holds, by their rows: their sums pass through the workspace."""
    counts, i, o = case
    g = gen(i + o)
    offsets, rows, row_token = layout(counts, g, sum(counts) // 2 if gather else None)
    x = normal(rows // 2 if gather else rows, i, dtype, g)
    w = padded(len(counts) * o, i, dtype, 0.0).unflatten(0, (len(counts), o))
    return offsets, rows, row_token, x, w, normal(rows, o, dtype, g)


def weight_buffers(case):
    counts, i, o = case
    return (torch.full((len(counts), o, (i + 3) // 4 * 4 + 4), float("nan"), device="cuda")[..., :i],
            torch.full((len(counts), o), float("nan"), device="cuda"))


# rows of every expert, in, out: pieces end inside steps of 64 rows, tiles inside the matrix; 263 and 1000 wide take
# tiles of 256 columns, 100 those of 128
CUT = [
    ([9001, 0, 4097, 63], 263, 515),
    ([9001, 0, 4097, 63], 1000, 515),
    ([1, 20011, 3073, 0, 3072], 100, 130),
    ([6145] * 9, 520, 260),
]


@pytest.mark.parametrize("case", CUT, ids=lambda c: f"{max(c[0])}r-{c[1]}-{c[2]}")
@pytest.mark.parametrize("gather", [False, True], ids=["in-order", "gathered"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_gradients_of_experts_that_are_cut(gs, case, gather, dtype):  # noqa: F811
    offsets, rows, row_token, x, w, dz = cut_inputs(case, gather, dtype)
    dw, db = weight_buffers(case)
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw, db=db, row_token=row_token)
    xs, zs = of_rows(x, row_token), dz.double()
    for e, r in segments(offsets):
        n, xe, ze = r.stop - r.start, xs[r].double(), zs[r]
        # a chain ends after 768 rows and the chains are added in float, so the length in the bound is that of a chain
        # and the number of chains
        room = (min(n, 768) + n // 768 + 8) * 2.0 ** -23
        close(dw[e], ze.T @ xe, room * (ze.abs().T @ xe.abs()) + 1e-30)
        close(db[e], ze.sum(0), room * ze.abs().sum(0) + 1e-30)
    beside = torch.as_strided(dw, (dw.shape[0] * dw.shape[1], dw.stride(1) - dw.shape[2]), (dw.stride(1), 1), dw.shape[2])
    assert torch.isnan(beside).all()
    for with_db in (True, False, True):
        again = weight_buffers(case)
        gs.expert_linear_backward(dz, x, w, offsets, dw=again[0], db=again[1] if with_db else None, row_token=row_token)
        assert torch.equal(again[0], dw) and (not with_db or torch.equal(again[1], db))
    assert gs.device_status() == 0


def test_workspace_belongs_to_the_stream_that_uses_it(gs, monkeypatch):  # noqa: F811
    case = ([9001, 0, 4097, 63], 263, 515)
    offsets, rows, _, x, w, dz = cut_inputs(case, False, BF16)
    side, taken = torch.cuda.Stream(), []
    empty = torch.empty

    def recorded(*args, **kwargs):
        taken.append((torch.cuda.current_stream().cuda_stream, kwargs.get("device")))
        return empty(*args, **kwargs)
    dw, db = weight_buffers(case)
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", recorded)
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw, db=db)
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw, db=db, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw, db=db, stream=side)
    monkeypatch.undo()
    torch.cuda.synchronize()
    here = torch.cuda.current_stream().cuda_stream
    assert [s for s, _ in taken] == [here, here, side.cuda_stream]


def test_gradients_on_two_streams_at_once(gs):  # noqa: F811
    """One gradient after the other on the current and a side stream, nothing waited for: as one by one."""
    case = ([9001, 0, 4097, 63], 263, 515)
    offsets, rows, _, x, w, dz = cut_inputs(case, False, BF16)
    other = normal(rows, case[2], BF16, gen(2))
    want = [weight_buffers(case) for _ in range(2)]
    for d, (dw, db) in zip((dz, other), want):
        gs.expert_linear_backward(d, x, w, offsets, dw=dw, db=db)
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [[weight_buffers(case) for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    for a, b in zip(*got):
        gs.expert_linear_backward(dz, x, w, offsets, dw=a[0], db=a[1])
        gs.expert_linear_backward(other, x, w, offsets, dw=b[0], db=b[1], stream=side)
    torch.cuda.synchronize()
    for mine, ref in zip(got, want):
        for dw, db in mine:
            assert torch.equal(dw, ref[0]) and torch.equal(db, ref[1])
    assert gs.device_status() == 0
