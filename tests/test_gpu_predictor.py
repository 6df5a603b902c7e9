"""The length predictor of examples/predict_and_route.py: its gradients against automatic
differentiation of the same network, and a short training run."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("predict_and_route", os.path.join(ROOT, "examples", "predict_and_route.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("top_k", [2, 9])
def test_gradients_of_the_whole_network(example, top_k):
    from paper_2605_16867_b200 import GoodServe
    gs = GoodServe(0)
    p = example.LengthPredictor(gs, features=40, gate_hidden=24, hidden=(33, 16, 8), top_k=top_k, seed=3)
    for layer in p.layers:                                    # masters equal to their 16-bit operands
        layer.master.copy_(layer.w)
    x, _, length = example.requests(500, 40, 1, gs.device)
    pred = p.forward(x)
    d = example._matrix(*pred.shape, gs.device, torch.float32)
    d.copy_(torch.randn(pred.shape, device=gs.device) / 500)
    p.backward(d)
    # the same network in 64 bits with the same choice of experts
    expert = p.kept[4]["expert"].long()
    ws = [[layer.master.double().requires_grad_(), layer.b.double().requires_grad_()] for layer in p.layers]

    def linear(h, wb, relu):
        """A layer whose answer is held in 16 bits, as the example holds it (the rounding has slope one)."""
        z = torch.einsum("eni,eoi->eno", h, wb[0]) + wb[1][:, None]
        z = torch.relu(z) if relu else z
        return z + (z.to(torch.bfloat16).double() - z).detach()
    h = x.double()[None]
    logits = linear(linear(h, ws[0], True), ws[1], False)[0]
    s = torch.softmax(logits, 1).gather(1, expert)
    weight = s / s.sum(1, keepdim=True)
    y = h.expand(9, -1, -1)
    for depth, wb in enumerate(ws[2:]):
        y = linear(y, wb, depth < 3)
    want = (weight * y[:, :, 0].T.gather(1, expert)).sum(1)
    (want * d[:, 0].double()).sum().backward()
    # 16-bit gradients between four layers: a few units of 2^-8 of the whole
    assert float((pred[:, 0].double() - want).detach().norm() / want.detach().norm()) < 2.0 ** -5
    for layer, (w, b) in zip(p.layers, ws):
        for got, ref in ((layer.dw, w.grad), (layer.db, b.grad)):
            off = float((got.double() - ref).norm() / ref.norm())
            print(tuple(got.shape), off)
            assert off < 2.0 ** -4
    assert gs.device_status() == 0
    gs.close()


def test_training_and_routing(example, capsys):
    losses, same = example.main(steps=60, batch=2048, top_k=3)
    assert sum(losses[-5:]) / 5 < 0.25 * losses[0]
    assert 0.0 <= same <= 1.0
    assert "device status 0" in capsys.readouterr().out
