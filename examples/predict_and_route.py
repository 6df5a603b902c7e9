"""A decode-length predictor on the library's operators, trained for a few steps and put in front of
the router.

The predictor is the mixture of Sec. 3.2: a two-layer gate over K experts, each a four-layer MLP; the
answer is the gate-weighted sum of the experts' answers (here the logarithm of the length).  top_k = K
is the paper's dense mixture, a smaller top_k asks the best experts alone.  All products, the routing,
the mixing and the clipping of the gradients are gs_* calls, forward and backward; PyTorch holds the
memory and takes Adam's elementwise step.

    python examples/predict_and_route.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import workloads as W  # noqa: E402
from paper_2605_16867_b200 import ExpertRouter, GoodServe, InstancePool  # noqa: E402

BF16 = torch.bfloat16


def _matrix(rows, cols, device, dtype=BF16):
    """Rows that start 16-byte aligned, whatever their width."""
    pad = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.zeros(rows, (cols + pad - 1) // pad * pad, dtype=dtype, device=device)[:, :cols]


class Layer:
    """Weights of one layer of all experts: float masters, 16-bit operands, float gradients."""

    def __init__(self, n_experts, fan_in, fan_out, generator, device):
        shape = (n_experts, fan_out)
        self.w = _matrix(n_experts * fan_out, fan_in, device).unflatten(0, shape)
        self.dw = _matrix(n_experts * fan_out, fan_in, device, torch.float32).unflatten(0, shape)
        self.master = torch.randn(*shape, fan_in, generator=generator, device=device) * (2.0 / fan_in) ** 0.5
        self.b, self.db = torch.zeros(shape, device=device), torch.zeros(shape, device=device)
        self.refresh()

    def refresh(self):
        self.w.copy_(self.master)

    def gradients(self):
        """The gradients' buffers whole, padding included (it stays zero)."""
        rows = self.dw.shape[0] * self.dw.shape[1]
        return [torch.as_strided(self.dw, (rows, self.dw.stride(1)), (self.dw.stride(1), 1)), self.db]


class LengthPredictor:
    def __init__(self, gs: GoodServe, features=256, n_experts=9, top_k=9, gate_hidden=128, hidden=(256, 128, 64), seed=0):
        g = torch.Generator(device=gs.device)
        g.manual_seed(seed)
        self.gs, self.features = gs, features
        self.router = ExpertRouter(n_experts, top_k)
        sizes = (features, *hidden, 1)
        self.gate = [Layer(1, features, gate_hidden, g, gs.device), Layer(1, gate_hidden, n_experts, g, gs.device)]
        self.experts = [Layer(n_experts, i, o, g, gs.device) for i, o in zip(sizes[:-1], sizes[1:])]
        self.layers = self.gate + self.experts
        self.moments = [(torch.zeros_like(p), torch.zeros_like(p)) for layer in self.layers for p in (layer.master, layer.b)]
        self.norm, self.steps = torch.zeros(1, device=gs.device), 0

    def forward(self, x):
        """Predicted log length [n, 1] in float; keeps what the gradients need."""
        gs, dev, n, k, e = self.gs, self.gs.device, x.shape[0], self.router.top_k, self.router.n_experts
        everyone = torch.tensor([0, n], dtype=torch.int32, device=dev)      # one expert that holds all rows: a plain layer
        g = _matrix(n, self.gate[0].w.shape[1], dev)
        logits = _matrix(n, e, dev)
        gs.expert_linear(x, self.gate[0].w, everyone, g, bias=self.gate[0].b, relu=True)
        gs.expert_linear(g, self.gate[1].w, everyone, logits, bias=self.gate[1].b)
        i32 = dict(dtype=torch.int32, device=dev)
        choice = dict(expert=torch.empty(n, k, **i32), weight=torch.empty(n, k, device=dev), offsets=torch.empty(e + 1, **i32),
                      row_token=torch.empty(n * k, **i32), token_row=torch.empty(n, k, **i32))
        gs.expert_route(logits, self.router, *choice.values())
        h, rows = [], choice["row_token"]
        for depth, layer in enumerate(self.experts):
            out = _matrix(n * k, layer.w.shape[1], dev)
            gs.expert_linear(h[-1] if h else x, layer.w, choice["offsets"], out, bias=layer.b,
                             row_token=None if h else rows, relu=depth + 1 < len(self.experts))
            h.append(out)
        pred = _matrix(n, 1, dev, torch.float32)
        gs.expert_combine(h[-1], choice["token_row"], pred, weight=choice["weight"])
        self.kept = (x, everyone, g, logits, choice, h)
        return pred

    def backward(self, d_pred):
        """Fills every layer's dw and db from the gradient of the prediction."""
        gs, dev = self.gs, self.gs.device
        x, everyone, g, logits, choice, h = self.kept
        d, d_weight = _matrix(*h[-1].shape, dev), torch.empty_like(choice["weight"])
        gs.expert_combine_backward(d_pred, h[-1], choice["token_row"], dy=d, weight=choice["weight"], d_weight=d_weight)
        for depth in reversed(range(len(self.experts))):
            layer, first = self.experts[depth], depth == 0
            below = None if first else _matrix(*h[depth - 1].shape, dev)
            gs.expert_linear_backward(d, x if first else h[depth - 1], layer.w, choice["offsets"], dx=below, dw=layer.dw,
                                      db=layer.db, row_token=choice["row_token"] if first else None, relu_input=not first)
            d = below
        d_logits, dg = _matrix(*logits.shape, dev), _matrix(*g.shape, dev)
        gs.expert_route_backward(logits, self.router, choice["expert"], d_weight, d_logits)
        gs.expert_linear_backward(d_logits, g, self.gate[1].w, everyone, dx=dg, dw=self.gate[1].dw, db=self.gate[1].db, relu_input=True)
        gs.expert_linear_backward(dg, x, self.gate[0].w, everyone, dw=self.gate[0].dw, db=self.gate[0].db)

    def step(self, x, target, rate=2e-3, max_norm=1.0):
        """One training step on the squared error of the log length; returns the loss (on the device)."""
        pred = self.forward(x)
        error = pred - target[:, None]
        d_pred = _matrix(*pred.shape, self.gs.device, torch.float32)
        d_pred.copy_(error * (2.0 / len(x)))
        self.backward(d_pred)
        self.gs.clip_grad_norm([t for layer in self.layers for t in layer.gradients()], max_norm, self.norm)
        self.steps += 1
        grads = [(p, t) for layer in self.layers for p, t in ((layer.master, layer.dw), (layer.b, layer.db))]
        for (p, t), (m, v) in zip(grads, self.moments):
            m.lerp_(t, 0.1)
            v.lerp_(t * t, 0.01)
            p.sub_(rate * (m / (1 - 0.9 ** self.steps)) / ((v / (1 - 0.99 ** self.steps)).sqrt() + 1e-8))
        for layer in self.layers:
            layer.refresh()
        return error.square().mean()

    def lengths(self, x):
        """pred_decode_len for the router: int32, in the range of the workloads."""
        return self.forward(x)[:, 0].exp().round().clamp(8, 8192).to(torch.int32)


def requests(n, features, seed, device):
    """Feature vectors whose application class and prompt length say something about the decode length."""
    rng = np.random.default_rng(seed)
    mixing = np.random.default_rng(99).normal(size=(12, features)) / 3
    kind, prompt = rng.integers(0, 9, n), np.clip(rng.lognormal(6.5, 1, n), 16, 16384)
    facts = np.concatenate([np.eye(9)[kind], np.log(prompt)[:, None] / 6, rng.normal(size=(n, 2)) * 0.3], 1)
    length = np.clip(np.exp(3.5 + 0.35 * kind + 0.1 * np.log(prompt) * (kind % 3) + 0.2 * rng.normal(size=n)), 8, 8192)
    x = _matrix(n, features, device)
    x.copy_(torch.from_numpy(facts @ mixing).to(device))
    return x, torch.from_numpy(prompt.astype(np.int32)).to(device), torch.from_numpy(length.astype(np.float32)).to(device)


def main(steps=150, batch=4096, top_k=9):
    gs = GoodServe(0)
    predictor = LengthPredictor(gs, top_k=top_k)
    losses = []
    for k in range(steps):
        x, _, length = requests(batch, predictor.features, k, gs.device)
        losses.append(predictor.step(x, length.log()))
        if k % 25 == 0 or k + 1 == steps:
            print(f"step {k:4d}  squared error of the log length {float(losses[-1]):.4f}  gradient norm {float(predictor.norm):.3f}")

    wl = W.make_workload(1, n_requests=16, n_active=16)
    pool = InstancePool.from_host(wl.types, wl.instances, gs.device)
    x, prompt, length = requests(65536, predictor.features, 10 ** 6, gs.device)
    slo = torch.full((len(x),), 20000.0, device=gs.device)
    found = {}
    for name, decode in (("predicted lengths", predictor.lengths(x)), ("true lengths", length.to(torch.int32))):
        out = [torch.empty(len(x), dtype=t, device=gs.device) for t in (torch.int32, torch.float32, torch.float32, torch.uint8)]
        gs.route_batch(prompt, decode, slo, pool, wl.ema_alpha, *out)
        found[name] = out[0]
        tiers = torch.bincount(out[3].long(), minlength=4).tolist()
        print(f"{name}: just-enough {tiers[1]}, fallback {tiers[2]} / {tiers[3]}")
    same = float((found["predicted lengths"] == found["true lengths"]).float().mean())
    print(f"the same instance for {100 * same:.1f} % of the requests; device status {gs.device_status()}")
    gs.close()
    return [float(v) for v in losses], same


if __name__ == "__main__":
    main()
