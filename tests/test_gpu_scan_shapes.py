"""The gated recurrence in every shape of its kernel: what the tests of one shape hold has to hold for all of them.

The shape goes by the sequences' average length and number: up to two rows a thread per four columns (forwards), up to eight a
thread per two, up to 64 four warps a sequence, then 8 or 16 warps and, with few sequences, clusters of up to eight thread
blocks along each of them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import (BAD_VALUE, BF16, F16, F32, clean_status, close, gen, gs, normal, padded, reference_scan,  # noqa: E402, F401
                              reference_scan_gradient, rounding, scan_inputs)

INF = float("inf")
# lengths, features
SHAPES = {
    "a row or two": ([1, 2, 0, 1] * 30, 70),
    "up to a block": ([5, 8, 0, 3] * 10, 70),
    "four warps": ([60, 0, 33, 17, 8, 64], 130),
    "wide": ([300] * 20 + [0, 77], 1000),
    "clusters of two and four": ([700] * 3, 64 * 16),
    "clusters of eight": ([4100, 0, 5003], 72),
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_the_last_state_over_the_first(gs, shape, dtype):  # noqa: F811
    """out_last may be h0 itself: every thread block has read its state before any writes the next one over it."""
    lengths, features = SHAPES[shape]
    n, s = sum(lengths), len(lengths)
    x, gate, offsets, h0 = scan_inputs(lengths, features, dtype, 100 + features)
    gate.add_(4.0)                                # (much of the state stays to the end, so that a state read too late shows)
    out, last = padded(n, features, dtype), padded(s, features, F32)
    gs.gated_scan(x, gate, offsets, out=out, h0=h0, last=last)
    _, after, _, _, err, want, want_err = reference_scan(x, gate, lengths, h0)
    close(out, after, err + rounding(after, dtype))
    close(last, want, want_err + rounding(want, F32))
    for _ in range(20):
        over, again = padded(s, features, F32).copy_(h0), padded(n, features, dtype)
        gs.gated_scan(x, gate, offsets, out=again, h0=over, last=over)
        assert torch.equal(over, last) and torch.equal(again, out)
    assert gs.device_status() == 0


def test_kept_states_come_from_the_pool_of_their_stream(gs):  # noqa: F811
    """Memory given back by a program on a side stream goes to that stream's next call, not to another stream's."""
    side = torch.cuda.Stream()
    states = gs.gated_scan_states(70001, 3, 1003, stream=side)
    assert states.shape == (70001 // 8 + 3, 1003) and states.dtype is F32 and states.stride() == (1004, 1)
    at, size = states.data_ptr(), states.shape[0] * 1004
    del states
    here = gs.gated_scan_states(70001, 3, 1003)
    assert here.data_ptr() != at
    with torch.cuda.stream(side):
        assert torch.empty(size, device="cuda").data_ptr() == at


@pytest.mark.parametrize("lengths,features,dtype", [
    ([1] * 700 + [900] + [0] * 200, 33, BF16), ([0] * 500 + [333], 130, F32), ([3] * 90 + [700], 72, F16), ([20] * 9 + [2500] + [1] * 90, 66, BF16)])
def test_one_long_sequence_among_short_ones(gs, lengths, features, dtype):  # noqa: F811
    """The shape goes by the average: the longest sequence may be anything, forwards and backwards."""
    n, s = sum(lengths), len(lengths)
    x, gate, offsets, h0 = scan_inputs(lengths, features, dtype, n, extra=1)
    out, last, states = padded(n, features, dtype), padded(s, features, F32), gs.gated_scan_states(n, s, features)
    gs.gated_scan(x, gate, offsets, out=out, h0=h0, last=last, states=states)
    before, after, a, c, err, want, want_err = reference_scan(x, gate, lengths, h0)
    close(out, after, err + rounding(after, dtype))
    close(last, want, want_err + rounding(want, F32))
    d_out, d_last = normal(n, features, dtype, gen(8)), normal(s, features, F32, gen(9))
    dx, d_gate, d_h0 = padded(n, features, dtype), padded(n, features, dtype), padded(s, features, F32)
    gs.gated_scan_backward(x, gate, offsets, states, dx=dx, d_gate=d_gate, d_out=d_out, d_last=d_last, d_h0=d_h0)
    want = reference_scan_gradient(x, lengths, before, a, c, err, d_out, d_last)
    close(dx, want[0], want[3] + rounding(want[0], dtype))
    close(d_gate, want[1], want[4] + rounding(want[1], dtype))
    close(d_h0, want[2], want[5] + rounding(want[2], F32))
    assert gs.device_status() == 0


GUARD = 24                                        # rows before and behind a matrix that nothing may touch


def guarded(rows, cols, dtype):
    """(whole buffer, the matrix inside it): rows of NaN on both sides, columns of NaN between the rows."""
    whole = padded(rows + 2 * GUARD, cols, dtype, extra=2)
    return whole, whole[GUARD:GUARD + rows]


def untouched(whole, rows, cols):
    """What lies around the matrix is as it was."""
    ld = whole.stride(0)
    full = torch.as_strided(whole, (whole.shape[0], ld), (ld, 1), whole.storage_offset())
    inside = torch.zeros(full.shape, dtype=torch.bool, device="cuda")
    inside[GUARD:GUARD + rows, :cols] = True
    return bool(torch.isnan(full[~inside]).all())


WRONG = [[-7, 4, 10 ** 9], [30, 2, 7], [2 ** 31 - 1, -2 ** 31, 5], [5, 20, 3, 25], [-1, -5, -2 ** 31, 2 ** 31 - 1], [9, 9, 8, 8, 9]]


@pytest.mark.parametrize("offsets", WRONG, ids=str)
@pytest.mark.parametrize("n", [3, 11, 100, 1201])                    # by the average: a thread per four, per two columns, four warps, the wide shape
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_offsets_that_make_no_sense_write_nothing_else(gs, offsets, n, dtype):  # noqa: F811
    """Offsets are clamped to the rows and made ascending; rows of no sequence (here NaN) are neither read nor written."""
    f, s = 40, len(offsets) - 1
    begin = [min(max(o, 0), n) for o in offsets[:-1]]
    end = [max(min(max(o, 0), n), b) for o, b in zip(offsets[1:], begin)]
    covered = torch.zeros(n, dtype=torch.int32, device="cuda")
    for b, e in zip(begin, end):
        covered[b:e] += 1
    x, gate = normal(n, f, dtype, gen(14)), normal(n, f, dtype, gen(15))
    x[covered == 0], gate[covered == 0] = float("nan"), float("nan")
    h0, d_last, d_out = normal(s, f, F32, gen(16)), normal(s, f, F32, gen(17)), normal(n, f, dtype, gen(18))
    given = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    rows = dict(out=n, last=s, states=n // 8 + s, dx=n, d_gate=n, d_h0=s)
    made = {k: guarded(r, f, dtype if k in ("out", "dx", "d_gate") else F32) for k, r in rows.items()}
    of = {k: m for k, (_, m) in made.items()}
    gs.gated_scan(x, gate, given, out=of["out"], h0=h0, last=of["last"], states=of["states"])
    assert gs.device_status() == BAD_VALUE
    gs.gated_scan_backward(x, gate, given, of["states"], dx=of["dx"], d_gate=of["d_gate"], d_out=d_out, d_last=d_last, d_h0=of["d_h0"])
    assert gs.device_status() == BAD_VALUE
    for k, (whole, _) in made.items():
        assert untouched(whole, rows[k], f), k
    for k in ("out", "dx", "d_gate"):
        assert torch.isnan(of[k][covered == 0]).all() and torch.isfinite(of[k][covered > 0].float()).all(), k
    assert torch.isfinite(of["last"]).all() and torch.isfinite(of["d_h0"]).all()
    for k, (b, e) in enumerate(zip(begin, end)):     # each sequence as if it were alone; rows of two hold either's values
        _, after, _, _, err, want, want_err = reference_scan(x[b:e], gate[b:e], [e - b], h0[k:k + 1])
        close(of["last"][k:k + 1], want, want_err + rounding(want, F32))
        alone = covered[b:e] == 1
        close(of["out"][b:e][alone], after[alone], (err + rounding(after, dtype))[alone])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_nothing_observed_in_sixteen_bits(gs, shape, dtype):  # noqa: F811
    """A gate of +infinity keeps the state whatever x holds there, one of -infinity replaces it but for 2^-125 of it; a column
    with a NaN among its gates has no say in the others."""
    lengths, features = SHAPES[shape]
    n, s = sum(lengths), len(lengths)
    x, gate, offsets, h0 = scan_inputs(lengths, features, dtype, 200 + features)
    g = gen(10)
    kind = torch.rand(n, features, generator=g, device="cuda")
    missing, fresh = kind < 0.3, (kind > 0.3) & (kind < 0.4)
    gate[missing], gate[fresh] = INF, -INF
    x[missing] = torch.where(torch.rand(n, features, generator=g, device="cuda") < 0.5, float("nan"), INF).to(dtype)[missing]
    for k in range(1, features, 11):              # (a column of its own each)
        gate[n // 2, k], x[n // 2, k] = float("nan"), 1.0
    sound = [k for k in range(features) if k % 11 != 1]
    out, last, states = padded(n, features, dtype), padded(s, features, F32), gs.gated_scan_states(n, s, features)
    gs.gated_scan(x, gate, offsets, out=out, h0=h0, last=last, states=states)
    d_out, d_last = normal(n, features, dtype, g), normal(s, features, F32, g)
    dx, d_gate, d_h0 = padded(n, features, dtype), padded(n, features, dtype), padded(s, features, F32)
    gs.gated_scan_backward(x, gate, offsets, states, dx=dx, d_gate=d_gate, d_out=d_out, d_last=d_last, d_h0=d_h0)
    assert torch.isnan(out[n // 2, 1::11]).all()
    x, gate, h0, d_out, d_last, missing = (t[:, sound] for t in (x, gate, h0, d_out, d_last, missing))
    before, after, a, c, err, want, want_err = reference_scan(x, gate, lengths, h0)
    close(out[:, sound], after, err + rounding(after, dtype))
    close(last[:, sound], want, want_err + rounding(want, F32))
    want = reference_scan_gradient(torch.where(missing, 0.0, x), lengths, before, a, c, err, d_out, d_last)
    close(dx[:, sound], want[0], want[3] + rounding(want[0], dtype))
    close(d_gate[:, sound], want[1], want[4] + rounding(want[1], dtype) + 2.0 ** -115)
    close(d_h0[:, sound], want[2], want[5] + rounding(want[2], F32) + 2.0 ** -115)
    assert (dx[:, sound][missing] == 0).all() and (d_gate[:, sound][missing] == 0).all()
