"""The length predictor's operators where there is nothing, or next to nothing, to do."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operators import BF16, F16, F32, clean_status, gen, gs, normal, padded, rest  # noqa: E402, F401

I32 = dict(dtype=torch.int32, device="cuda")


def test_gradients_without_rows(gs):  # noqa: F811
    w = torch.zeros(3, 16, 24, dtype=BF16, device="cuda")
    offsets = torch.zeros(4, **I32)
    dz, x, dx = padded(0, 16, BF16), padded(0, 24, BF16), padded(0, 24, BF16)
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx)
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx, relu_input=True)
    dw, db = torch.full((3, 16, 24), 7.0, device="cuda"), torch.full((3, 16), 7.0, device="cuda")
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx, dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()
    # no tokens: nothing is written; tokens that all lost their rows: zeros
    y = normal(5, 24, BF16, gen(1))
    gs.expert_combine_backward(padded(0, 24, BF16), y, torch.zeros(0, 2, **I32), dy=padded(5, 24, BF16))
    gs.expert_combine_backward(padded(0, 24, BF16), y, torch.zeros(0, 2, **I32), d_weight=torch.zeros(0, 2, device="cuda"))
    none, lost = padded(0, 24, BF16), torch.full((4, 2), -1, **I32)
    gs.expert_combine_backward(normal(4, 24, BF16, gen(2)), none, lost, dy=none)
    d_weight = torch.full((4, 2), 7.0, device="cuda")
    gs.expert_combine_backward(normal(4, 24, BF16, gen(2)), none, lost, dy=none, d_weight=d_weight)
    out = torch.full((4, 24), 7.0, dtype=BF16, device="cuda")
    gs.expert_combine(none, lost, out)
    assert (d_weight == 0).all() and (out == 0).all()
    assert gs.device_status() == 0


@pytest.mark.parametrize("features", [1, 8, 40, 250, 256, 1000, 1024, 2500])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_combine_backward_writes_the_named_rows_alone(gs, features, dtype):  # noqa: F811
    n, k = 75, 3
    g = gen(features)
    rows = n * k + 20
    token_row = torch.randperm(rows, generator=g, device="cuda")[: n * k].view(n, k).to(torch.int32)
    token_row[torch.rand(n, k, generator=g, device="cuda") < 0.2] = -1
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[token_row[token_row >= 0].long()] = True
    y, weight = normal(rows, features, dtype, g), torch.randn(n, k, generator=g, device="cuda")
    for d_dtype in (dtype, F32):
        for relu in (False, True):
            dy = padded(rows, features, dtype, extra=1)
            gs.expert_combine_backward(normal(n, features, d_dtype, g), y, token_row, dy=dy, weight=weight, relu=relu)
            assert torch.isfinite(dy[named]).all()
            assert torch.isnan(dy[~named]).all()
            assert torch.isnan(rest(dy)).all()
    assert gs.device_status() == 0
