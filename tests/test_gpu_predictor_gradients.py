"""The length predictor of examples/predict_and_route.py against its formula in 64 bits, closely.

Layers' answers are held in bfloat16 on both sides, so the prediction differs only where a sum in float rounds
to the other neighbour (one value in some hundreds, by 2^-8 of itself): 2^-9 of the whole.  Gradients pass through up to
six roundings to bfloat16 (u = 2^-8 each, both ways at random) that the formula does not take: sqrt(6) u, and half
as much again twice over: 2^-6 of the whole."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_predictor import example  # noqa: E402, F401


def formula(layers, x, expert):
    """Prediction for this choice of experts, and the parameters it was made of, in 64 bits."""
    params = [[layer.master.double().requires_grad_(), layer.b.double().requires_grad_()] for layer in layers]

    def layer(h, wb, relu):
        z = torch.baddbmm(wb[1][:, None], h, wb[0].transpose(1, 2))
        z = z.clamp_min(0) if relu else z
        return z + (z.bfloat16().double() - z).detach()
    one = x.double()[None]
    logits = layer(layer(one, params[0], True), params[1], False)[0]
    score = torch.softmax(logits, 1).gather(1, expert)
    y = one.expand(logits.shape[1], -1, -1)
    for depth, wb in enumerate(params[2:], 3):
        y = layer(y, wb, depth < len(params))
    return (score / score.sum(1, keepdim=True) * y[:, :, 0].T.gather(1, expert)).sum(1), params


def apart(a, b):
    return float((a.double() - b.detach()).norm() / b.detach().norm())


@pytest.mark.parametrize("top_k,hidden,rows", [(9, (256, 128, 64), 2000), (4, (40, 24, 8), 777), (1, (64,), 300)])
def test_prediction_and_gradients(example, top_k, hidden, rows):  # noqa: F811
    from paper_2605_16867_b200 import GoodServe
    gs = GoodServe(0)
    p = example.LengthPredictor(gs, features=96, gate_hidden=48, hidden=hidden, top_k=top_k, seed=5)
    for layer in p.layers:
        layer.master.copy_(layer.w)
    x, _, _ = example.requests(rows, 96, 2, gs.device)
    pred = p.forward(x)
    d = example._matrix(*pred.shape, gs.device, torch.float32)
    d.copy_(torch.randn(pred.shape, generator=torch.Generator("cuda").manual_seed(3), device=gs.device) / rows)
    p.backward(d)
    want, params = formula(p.layers, x, p.kept[4]["expert"].long())
    (want * d[:, 0].double()).sum().backward()
    assert apart(pred[:, 0], want) < 2.0 ** -9
    for depth, (layer, (w, b)) in enumerate(zip(p.layers, params)):
        if top_k == 1 and depth < 2:                          # one weight of one: the gate has no gradient
            assert float(layer.dw.abs().max()) < 1e-6
            continue
        assert apart(layer.dw, w.grad) < 2.0 ** -6 and apart(layer.db, b.grad) < 2.0 ** -6, depth
    assert gs.device_status() == 0
    gs.close()
