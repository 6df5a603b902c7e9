"""The gated recurrence in every shape of its kernel: what the tests of one shape hold has to hold for all of them.

The shape goes by the sequences' average length and number: up to two rows a thread per four columns (forwards), up to eight a
thread per two, up to 64 four warps a sequence, then 8 or 16 warps and, with few sequences, clusters of up to eight thread
blocks along each of them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import BF16, F16, F32, clean_status, close, gs, padded, reference_scan, rounding, scan_inputs  # noqa: E402, F401

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
