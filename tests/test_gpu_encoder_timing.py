"""Which kernel the time of the encoder's operators is booked under, and how many launches each call makes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import BF16, F32, gen, gs, normal, padded  # noqa: E402, F401

EXPERT_LINEAR, EMBEDDING, SCAN, DROPOUT, LINEAR, COUNT = 9, 12, 13, 14, 15, 16     # gs_kernel


def booked(gs, call):  # noqa: F811
    """Launches by kernel of one call."""
    gs.timing_enable(True)
    call()
    torch.cuda.synchronize()
    launches = {}
    for k in range(COUNT):
        ms, n = gs.timing_read(k)
        if n:
            launches[k] = n
            assert ms > 0
    gs.timing_enable(False)
    return launches


def test_dense_layers_are_booked_as_such(gs):  # noqa: F811
    g = gen(1)
    for rows in (5, 300, 20000):                  # (where the weights' gradient is cut into pieces, another launch adds them up)
        x, w, dz = normal(rows, 128, BF16, g), normal(64, 128, BF16, g), normal(rows, 64, BF16, g)
        out, dx, dw, db = padded(rows, 64, BF16), padded(rows, 128, BF16), padded(64, 128, F32), torch.empty(64, device="cuda")
        assert booked(gs, lambda: gs.linear(x, w, out)) == {LINEAR: 1}
        assert booked(gs, lambda: gs.linear_backward(dz, x, w, dx=dx)) == {LINEAR: 1}
        launches = booked(gs, lambda: gs.linear_backward(dz, x, w, dx=dx, dw=dw, db=db))
        assert launches == {LINEAR: 3 if gs._lib.gs_linear_backward_workspace(gs._h, rows, 128, 64) > 0 else 2}
        assert booked(gs, lambda: gs.activation_backward(dz, out, "relu", dz)) == {LINEAR: 1}
        # the experts' products stay under their own
        offsets, we = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), w.unflatten(0, (1, 64))
        assert set(booked(gs, lambda: gs.expert_linear_backward(dz, x, we, offsets, dx=dx, dw=dw.unflatten(0, (1, 64))))) == {EXPERT_LINEAR}


def test_the_others_are_booked_under_theirs(gs):  # noqa: F811
    g = gen(2)
    table, ids = normal(50, 40, BF16, g), torch.arange(30, dtype=torch.int32, device="cuda")
    e, d_table = padded(30, 40, BF16), padded(50, 40, F32)
    assert booked(gs, lambda: gs.embedding(table, ids, e)) == {EMBEDDING: 1}
    assert set(booked(gs, lambda: gs.embedding_backward(e, ids, d_table))) == {EMBEDDING}
    offsets, out = torch.tensor([0, 30], dtype=torch.int32, device="cuda"), padded(30, 40, BF16)
    states = gs.gated_scan_states(30, 1, 40)
    assert booked(gs, lambda: gs.gated_scan(e, e, offsets, out=out, states=states)) == {SCAN: 1}
    assert booked(gs, lambda: gs.gated_scan_backward(e, e, offsets, states, dx=out, d_out=e)) == {SCAN: 1}
    assert booked(gs, lambda: gs.dropout(e, torch.zeros(2, dtype=torch.int64, device="cuda"), 0.1, out)) == {DROPOUT: 1}
