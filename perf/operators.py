"""What is measured of the length predictor's operators: routing of requests to experts, the
experts' products, the weighted sum of what they return, each with its gradient, and the clipping
of the gradients by their global norm.

``own`` false: the plain form, elementary torch operations in 32 bits.  ``own`` true: the calls a
user makes of the library.  ``prepare`` makes inputs and the output buffers that a program keeps.
"""
import functools
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_DEV = "cuda"
_LARGEST = 3.4028234663852886e38


def listed():
    return [
        # a quiet scheduling tick: 256 requests, nine length classes, the two best mixed (latency)
        dict(name="route 256 x 9 top 2", op="route", tokens=256, experts=9, top_k=2, score="softmax", groups=1,
             top_groups=1, group_top=1, renorm=True, bias=False, masked=False, type="f32", grad=False),
        # a full round of 1,048,576 pending requests over the same nine classes, some of them switched off
        dict(name="route 1048576 x 9 top 2", op="route", tokens=1048576, experts=9, top_k=2, score="softmax",
             groups=1, top_groups=1, group_top=1, renorm=True, bias=False, masked=True, type="f32", grad=False),
        # a training batch over many fine experts: sigmoid scores, balance bias, groups; with the gradient
        dict(name="route 131072 x 256 grouped + grad", op="route", tokens=131072, experts=256, top_k=8,
             score="sigmoid", groups=8, top_groups=4, group_top=2, renorm=True, bias=True, masked=False, type="bf16",
             grad=True),
        # the quiet tick's first layer: the weights' read is what counts
        dict(name="product 256 requests", op="product", tokens=256, experts=9, top_k=2, fan_in=2048, fan_out=1024,
             gather=True, relu=True, type="bf16"),
        # a round's first layer
        dict(name="product 131072 requests", op="product", tokens=131072, experts=9, top_k=2, fan_in=2048,
             fan_out=1024, gather=True, relu=True, type="bf16"),
        # odd sizes, sixteen uneven experts, a later layer without activation
        dict(name="product 20011 x 1000 to 500", op="product", tokens=20011, experts=16, top_k=3, fan_in=1000,
             fan_out=500, gather=False, relu=False, type="f16"),
        # training, a later layer: gradients of input, weights and bias, the layer below being a ReLU
        dict(name="product grad 16384", op="product_grad", tokens=16384, experts=9, top_k=2, fan_in=1024,
             fan_out=512, gather=False, relu=True, dx=True, type="f16"),
        # training, the first layer: weights and bias alone
        dict(name="product grad 65536 first layer", op="product_grad", tokens=65536, experts=9, top_k=2,
             fan_in=2048, fan_out=1024, gather=True, relu=False, dx=False, type="bf16"),
        # the experts' answers of a round, weighted and summed per request
        dict(name="combine 131072 x 1024", op="combine", tokens=131072, experts=9, top_k=2, features=1024,
             type="bf16", grad=False),
        # ... and back in training
        dict(name="combine grad 65536 x 1024", op="combine", tokens=65536, experts=9, top_k=2, features=1024,
             type="bf16", grad=True),
        # gradients of a small predictor, odd sizes (latency)
        dict(name="clip 8 tensors 0.2 M", op="clip", tensors=8, elements=200001, type="f32", norm=1.0),
        # gradients of a large one, weights in 16 bits and the rest in 32
        dict(name="clip 48 tensors 268 M", op="clip", tensors=48, elements=268435456, type="mixed", norm=1.0),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["route", "route", "product", "product", "product_grad", "product_grad", "combine", "clip"])
    if op == "route":
        grad = rng.random() < 0.5
        if rng.random() < 0.5:                       # few length classes
            experts, groups, top_groups, group_top = rng.randint(4, 33), 1, 1, 1
            score, bias = "softmax", False
        else:                                        # many fine experts
            groups = rng.choice([1, 2, 4, 8, 16])
            experts = groups * rng.randint(max(2, 32 // groups), 256 // groups)
            top_groups = rng.randint((groups + 1) // 2, groups)
            group_top = rng.randint(1, 2)
            score, bias = rng.choice(["softmax", "sigmoid"]), rng.random() < 0.7
        top_k = rng.randint(1, min(8, experts * top_groups // groups))
        tokens = _log_int(rng, 200, min(1048576, 33554432 // experts))
        return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, score=score, groups=groups,
                    top_groups=top_groups, group_top=group_top, bias=bias, masked=rng.random() < 0.3,
                    renorm=top_k > 1 and rng.random() < 0.7, type=rng.choice(["f32", "bf16", "f16"]), grad=grad)
    if op in ("product", "product_grad"):
        experts, top_k = rng.randint(4, 64), rng.randint(1, 4)
        fan_in, fan_out = _log_int(rng, 64, 2048), _log_int(rng, 64, 2048)
        if rng.random() < 0.15:
            fan_out = 1                              # the last layer of an expert
        per_token = 2.0 * top_k * fan_in * fan_out * (2 if op == "product_grad" else 1)
        most = int(min(131072, 1.0e12 / per_token, 5.0e8 / (top_k * (fan_in + fan_out))))
        case = dict(op=op, tokens=_log_int(rng, 200, max(201, most)), experts=experts, top_k=top_k, fan_in=fan_in,
                    fan_out=fan_out, gather=rng.random() < 0.5, relu=rng.random() < 0.5,
                    type=rng.choice(["bf16", "f16"]))
        if op == "product_grad":
            case["dx"] = rng.random() < 0.7
        return case
    if op == "combine":
        features, top_k = _log_int(rng, 1, 4096), rng.randint(1, 8)
        tokens = _log_int(rng, 200, int(max(201, min(262144, 3.0e8 / ((features + 8) * top_k)))))
        return dict(op=op, tokens=tokens, experts=rng.randint(4, 64), top_k=top_k, features=features,
                    type=rng.choice(["bf16", "f16"]), grad=rng.random() < 0.5)
    return dict(op="clip", tensors=rng.randint(1, 60), elements=_log_int(rng, 100000, 200000000),
                type=rng.choice(["f32", "bf16", "f16", "mixed"]), norm=rng.choice([0.5, 1.0, 1.0e4]))


# ---- inputs ---------------------------------------------------------------------------------

def _generator(case, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _padded(rows, cols, dtype):
    """Rows that start 16-byte aligned, as the library wants them: [rows, cols] of a wider buffer."""
    ld = (cols + 7) // 8 * 8
    return torch.zeros(rows, ld, dtype=dtype, device=_DEV)[:, :cols]


def _normal(rows, cols, dtype, g, scale):
    out = _padded(rows, cols, dtype)
    out.copy_(torch.randn(rows, cols, generator=g, device=_DEV) * scale)
    return out


def _popularity(experts, g):
    """How much likelier some experts are than others: the loads differ by a factor of ten or so."""
    return torch.randn(experts, generator=g, device=_DEV) * 0.8


def _close(values, err):
    """Rows where two neighbours of the descending values are nearer than what 32 bits tell apart
    (equal ones are fine: they go to the lower index)."""
    gap = values[:, :-1] - values[:, 1:]
    return ((gap > 0) & (gap < err[:, :-1] + err[:, 1:])).any(1)


def _near_ties(case, logits, bias):
    """Rows whose choice hangs on the last bits of a score; they are drawn again."""
    x = logits.double()
    on = x > -math.inf
    s = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(torch.where(on.any(1, keepdim=True), x, 0.0), 1)
    c = s + bias.double() if bias is not None else s
    err = 1e-6 * (s + c.abs())
    c = torch.where(on, c, -4.0)
    near = torch.zeros(len(c), dtype=torch.bool, device=c.device)
    if case["groups"] > 1:
        parts = c.view(len(c), case["groups"], -1)
        best, at = parts.sort(dim=2, descending=True, stable=True)
        best, off = best[:, :, :case["group_top"]], err.view_as(parts).gather(2, at)[:, :, :case["group_top"]].sum(2)
        best = torch.where(best > -3.0, best, 0.0).sum(2)
        best, at = best.sort(dim=1, descending=True, stable=True)
        off, cut = off.gather(1, at), slice(case["top_groups"] - 1, case["top_groups"] + 1)
        near = _close(best[:, cut], off[:, cut])
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, at[:, :case["top_groups"]], True)
        c = torch.where(keep[:, :, None], parts, -4.0).view_as(c)
    c, at = c.sort(dim=1, descending=True, stable=True)
    return near | _close(c[:, :case["top_k"] + 1], err.gather(1, at)[:, :case["top_k"] + 1])


def _some_logits(case, n, popularity, g):
    x = torch.randn(n, case["experts"], generator=g, device=_DEV) * 1.5 + popularity
    if case["masked"]:                              # classes switched off, and requests with none left at all
        x.masked_fill_(torch.rand(x.shape, generator=g, device=_DEV) < 0.05, -math.inf)
        x[torch.rand(n, generator=g, device=_DEV) < 0.002] = -math.inf
    return x.to(_TYPES[case["type"]])


def _prepare_route(case, g):
    n, e, k = case["tokens"], case["experts"], case["top_k"]
    popularity = _popularity(e, g)
    bias = torch.randn(e, generator=g, device=_DEV) * 0.05 if case["bias"] else None
    logits = _some_logits(case, n, popularity, g)
    bad = torch.cat([_near_ties(case, part, bias) for part in logits.split(131072)]).nonzero()[:, 0]
    while bad.numel():
        logits[bad] = _some_logits(case, bad.numel(), popularity, g)
        bad = bad[_near_ties(case, logits[bad], bias)]
    i32 = dict(dtype=torch.int32, device=_DEV)
    s = dict(logits=logits, bias=bias, expert=torch.empty(n, k, **i32),
             weight=torch.empty(n, k, dtype=torch.float32, device=_DEV), offsets=torch.empty(e + 1, **i32),
             row_token=torch.empty(n * k, **i32), token_row=torch.empty(n, k, **i32))
    if case["grad"]:
        s["d_weight"] = torch.randn(n, k, generator=g, device=_DEV) * 0.01
        s["d_logits"] = torch.empty_like(logits)
    return s


def _dispatch(case, g):
    """Which expert every request's slots went to, in the order that the products work in."""
    n, k, e = case["tokens"], case["top_k"], case["experts"]
    scores = torch.randn(n, e, generator=g, device=_DEV) + _popularity(e, g)
    expert = scores.topk(k, dim=1)[1]
    weight = torch.softmax(torch.randn(n, k, generator=g, device=_DEV), 1)
    order = torch.sort(expert.reshape(-1), stable=True)[1]
    row_token = (order // k).to(torch.int32)
    token_row = torch.empty_like(order)
    token_row[order] = torch.arange(n * k, device=_DEV)
    counts = torch.bincount(expert.reshape(-1), minlength=e)
    offsets = torch.zeros(e + 1, dtype=torch.int32, device=_DEV)
    offsets[1:] = counts.cumsum(0)
    return dict(weight=weight, row_token=row_token, token_row=token_row.view(n, k).to(torch.int32), offsets=offsets,
                bounds=offsets.tolist())


def _weights(case, g):
    e, o, i = case["experts"], case["fan_out"], case["fan_in"]
    return _normal(e * o, i, _TYPES[case["type"]], g, i ** -0.5).unflatten(0, (e, o))


def _prepare_product(case, g):
    t, rows = _TYPES[case["type"]], case["tokens"] * case["top_k"]
    s = _dispatch(case, g)
    s["x"] = _normal(case["tokens"] if case["gather"] else rows, case["fan_in"], t, g, 1.0)
    s["w"] = _weights(case, g)
    s["bias"] = torch.randn(case["experts"], case["fan_out"], generator=g, device=_DEV) * 0.1
    s["out"] = _padded(rows, case["fan_out"], t)
    return s


def _prepare_product_grad(case, g):
    t, rows = _TYPES[case["type"]], case["tokens"] * case["top_k"]
    s = _dispatch(case, g)
    s["x"] = _normal(case["tokens"] if case["gather"] else rows, case["fan_in"], t, g, 1.0)
    if case["relu"]:                                # the layer below answers with zeros where it was cut off
        s["x"].relu_()
    s["w"] = _weights(case, g)
    s["dz"] = _normal(rows, case["fan_out"], t, g, 0.05)
    s["dx"] = _padded(rows, case["fan_in"], t) if case["dx"] else None
    s["dw"] = torch.empty(case["experts"], case["fan_out"], (case["fan_in"] + 7) // 8 * 8, device=_DEV)[..., :case["fan_in"]]
    s["db"] = torch.empty(case["experts"], case["fan_out"], device=_DEV)
    return s


def _prepare_combine(case, g):
    t, rows = _TYPES[case["type"]], case["tokens"] * case["top_k"]
    s = _dispatch(case, g)
    s["y"] = _normal(rows, case["features"], t, g, 1.0)
    if case["grad"]:
        s["d_out"] = _normal(case["tokens"], case["features"], t, g, 0.05)
        s["dy"] = _padded(rows, case["features"], t)
        s["d_weight"] = torch.empty(case["tokens"], case["top_k"], device=_DEV)
    else:
        s["out"] = _padded(case["tokens"], case["features"], t)
    return s


def _clip_sizes(case):
    """Sizes of a model's gradients: a few matrices hold most of the elements, biases are small."""
    n, total = case["tensors"], case["elements"]
    shares = [1.0 / (1 + (3 * j) % 7) ** 2 if j % 2 == 0 else 1e-4 for j in range(n)]
    sizes = [max(1, int(total * s / sum(shares)) | (j & 1)) for j, s in enumerate(shares)]
    return sizes


def _clip_types(case):
    if case["type"] != "mixed":
        return [_TYPES[case["type"]]] * case["tensors"]
    return [torch.bfloat16 if j % 2 == 0 else torch.float32 for j in range(case["tensors"])]


def _prepare_clip(case, g):
    pairs = list(zip(_clip_sizes(case), _clip_types(case)))
    scale = 3.0 / math.sqrt(sum(n for n, _ in pairs))        # a global norm of about 3
    return dict(grads=[(torch.randn(n, generator=g, device=_DEV) * scale).to(t) for n, t in pairs],
                outs=[torch.empty(n, dtype=t, device=_DEV) for n, t in pairs],
                norm=torch.empty(1, dtype=torch.float32, device=_DEV))


def prepare(case, seed):
    g = _generator(case, seed)
    makers = dict(route=_prepare_route, product=_prepare_product, product_grad=_prepare_product_grad,
                  combine=_prepare_combine, clip=_prepare_clip)
    s = makers[case["op"]](case, g)
    s["case"] = case
    return s


# ---- plain forms ----------------------------------------------------------------------------

def _pick(c, k):
    """The k largest of every row in descending order, equal ones by index."""
    v, i = torch.sort(c, dim=1, descending=True, stable=True)
    return v[:, :k], i[:, :k]


def _scores(case, x):
    on = x > -math.inf
    if case["score"] == "sigmoid":
        return torch.where(on, 1.0 / (1.0 + torch.exp(-x)), 0.0), on
    top = x.amax(1, keepdim=True).clamp_min(-_LARGEST)
    p = torch.where(on, torch.exp(x - top), 0.0)
    return p / p.sum(1, keepdim=True).clamp_min(1e-30), on


def _plain_route(s):
    case, k, e = s["case"], s["case"]["top_k"], s["case"]["experts"]
    x = s["logits"].float().clamp_max(_LARGEST)
    score, on = _scores(case, x)
    choice = torch.where(on, score + s["bias"] if s["bias"] is not None else score, -math.inf)
    if case["groups"] > 1:
        parts = choice.view(len(choice), case["groups"], -1)
        best = torch.sort(parts, dim=2, descending=True)[0][:, :, :case["group_top"]]
        best = torch.where(best[:, :, 0] > -math.inf, torch.where(best > -math.inf, best, 0.0).sum(2), -math.inf)
        _, chosen = _pick(best, case["top_groups"])
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, chosen, True)
        choice = torch.where(keep[:, :, None], parts, -math.inf).view_as(choice)
    value, expert = _pick(choice, k)
    there = value > -math.inf
    picked = torch.where(there, score.gather(1, expert), 0.0)
    total = picked.sum(1, keepdim=True) + 1e-20
    weight = picked / total if case["renorm"] else picked
    expert = torch.where(there, expert, -1)
    flat = torch.where(there, expert, e).reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    counts = torch.bincount(flat, minlength=e + 1)[:e].cumsum(0)
    offsets = torch.cat([counts.new_zeros(1), counts])
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    real = torch.arange(order.numel(), device=order.device) < offsets[-1]
    out = dict(expert=expert.int(), weight=weight, offsets=offsets.int(),
               row_token=torch.where(real, order // k, -1).int(),
               token_row=torch.where(there, place.view_as(expert), -1).int())
    if case["grad"]:
        dw = torch.where(there, s["d_weight"], 0.0)
        d_picked = torch.where(there, (dw - (dw * weight).sum(1, keepdim=True)) / total, 0.0) if case["renorm"] else dw
        d_score = torch.zeros_like(score).scatter_add_(1, expert.clamp_min(0), d_picked)
        if case["score"] == "sigmoid":
            dx = d_score * score * (1.0 - score)
        else:
            dx = score * (d_score - (d_score * score).sum(1, keepdim=True))
        out["d_logits"] = dx.to(s["logits"].dtype)
    return out


def _segments(s):
    return [(e, a, b) for e, (a, b) in enumerate(zip(s["bounds"][:-1], s["bounds"][1:]))]


def _rows_of(s):
    x = s["x"].float()
    return x[s["row_token"].long()] if s["case"]["gather"] else x


def _plain_product(s):
    x, w = _rows_of(s), s["w"].float()
    z = torch.cat([x[a:b] @ w[e].T + s["bias"][e] for e, a, b in _segments(s)])
    return (torch.relu(z) if s["case"]["relu"] else z).to(s["x"].dtype)


def _plain_product_grad(s):
    x, w, dz = _rows_of(s), s["w"].float(), s["dz"].float()
    out = dict(dw=torch.stack([dz[a:b].T @ x[a:b] for _, a, b in _segments(s)]),
               db=torch.stack([dz[a:b].sum(0) for _, a, b in _segments(s)]))
    if s["case"]["dx"]:
        dx = torch.cat([dz[a:b] @ w[e] for e, a, b in _segments(s)])
        out["dx"] = (torch.where(x > 0, dx, 0.0) if s["case"]["relu"] else dx).to(s["x"].dtype)
    return out


def _plain_combine(s):
    rows = s["token_row"].long()
    y = s["y"].float()[rows]
    if not s["case"]["grad"]:
        return (y * s["weight"][:, :, None]).sum(1).to(s["y"].dtype)
    d_out = s["d_out"].float()
    dy = torch.empty(s["y"].shape, dtype=torch.float32, device=y.device)
    dy[rows.reshape(-1)] = (d_out[:, None, :] * s["weight"][:, :, None]).flatten(0, 1)
    return dict(dy=dy.to(s["y"].dtype), d_weight=(y * d_out[:, None, :]).sum(2))


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.where(torch.isfinite(norm), (s["case"]["norm"] / (norm + 1e-6)).clamp_max(1.0), 1.0)
    return dict(norm=norm.view(1), grads=[(g.float() * factor).to(g.dtype) for g in s["grads"]])


# ---- the library's operators ----------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _library():
    import paper_2605_16867_b200 as lib
    return lib, lib.GoodServe(torch.cuda.current_device())


@functools.lru_cache(maxsize=None)
def _router(experts, top_k, score, groups, top_groups, group_top, renorm):
    return _library()[0].ExpertRouter(experts, top_k, score=score, n_groups=groups, top_groups=top_groups,
                                      group_top=group_top, renormalise=renorm)


def _own_route(s):
    c, (_, gs) = s["case"], _library()
    router = _router(c["experts"], c["top_k"], c["score"], c["groups"], c["top_groups"], c["group_top"], c["renorm"])
    gs.expert_route(s["logits"], router, s["expert"], s["weight"], s["offsets"], s["row_token"], s["token_row"],
                    bias=s["bias"])
    out = {k: s[k] for k in ("expert", "weight", "offsets", "row_token", "token_row")}
    if c["grad"]:
        gs.expert_route_backward(s["logits"], router, s["expert"], s["d_weight"], s["d_logits"])
        out["d_logits"] = s["d_logits"]
    return out


def _own_product(s):
    c, (_, gs) = s["case"], _library()
    gs.expert_linear(s["x"], s["w"], s["offsets"], s["out"], bias=s["bias"],
                     row_token=s["row_token"] if c["gather"] else None, relu=c["relu"])
    return s["out"]


def _own_product_grad(s):
    c, (_, gs) = s["case"], _library()
    gs.expert_linear_backward(s["dz"], s["x"], s["w"], s["offsets"], dx=s["dx"], dw=s["dw"], db=s["db"],
                              row_token=s["row_token"] if c["gather"] else None, relu_input=c["relu"])
    return {k: s[k] for k in ("dw", "db", "dx") if s[k] is not None}


def _own_combine(s):
    _, gs = _library()
    if not s["case"]["grad"]:
        gs.expert_combine(s["y"], s["token_row"], s["out"], weight=s["weight"])
        return s["out"]
    gs.expert_combine_backward(s["d_out"], s["y"], s["token_row"], s["dy"], weight=s["weight"],
                               d_weight=s["d_weight"])
    return dict(dy=s["dy"], d_weight=s["d_weight"])


def _own_clip(s):
    _, gs = _library()
    gs.clip_grad_norm(s["grads"], s["case"]["norm"], s["norm"], outs=s["outs"])
    return dict(norm=s["norm"], grads=s["outs"])


_PLAIN = dict(route=_plain_route, product=_plain_product, product_grad=_plain_product_grad, combine=_plain_combine,
              clip=_plain_clip)
_OWN = dict(route=_own_route, product=_own_product, product_grad=_own_product_grad, combine=_own_combine,
            clip=_own_clip)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    op, width = case["op"], {"f32": 4, "bf16": 2, "f16": 2, "mixed": 2}[case["type"]]
    n = case.get("tokens", 0)
    if op == "route":
        k, e = case["top_k"], case["experts"]
        size = n * e * width + n * k * 16 + 4 * (e + 1) + (4 * e if case["bias"] else 0)
        flops = n * e * 4.0
        if case["grad"]:
            size += n * e * width + n * k * 4
            flops += n * e * 4.0
        return dict(bytes=size, flops=flops)
    if op in ("product", "product_grad"):
        e, k, i, o = case["experts"], case["top_k"], case["fan_in"], case["fan_out"]
        rows = n * k
        x = (n if case["gather"] else rows) * i * width + (4 * rows if case["gather"] else 0)
        if op == "product":
            return dict(bytes=x + e * o * (i * width + 4) + rows * o * width, flops=2.0 * rows * i * o)
        size, flops = x + rows * o * width + 4 * e * o * (i + 1), 2.0 * rows * i * o
        if case["dx"]:
            size, flops = size + rows * i * width + e * o * i * width, 2 * flops
        return dict(bytes=size, flops=flops)
    if op == "combine":
        k, f = case["top_k"], case["features"]
        size = n * f * width * (k + 1) + n * k * 8
        if case["grad"]:
            size += n * k * (f * width + 4)
        return dict(bytes=size, flops=2.0 * n * k * f * (2 if case["grad"] else 1))
    sizes = _clip_sizes(case)
    size = sum(2 * m * t.itemsize for m, t in zip(sizes, _clip_types(case)))
    return dict(bytes=size, flops=3.0 * sum(sizes))


# ---- the definitions in 64 bits ---------------------------------------------------------------

def _exact_route(case, s):
    """Definition, row block by row block: whole numbers are compared between the two forms."""
    weights, slopes = [], []
    k, groups = case["top_k"], case["groups"]
    for lo in range(0, case["tokens"], 131072):
        x = s["logits"][lo:lo + 131072].double()
        off = torch.isinf(x) & (x < 0)
        if case["score"] == "sigmoid":
            p = torch.sigmoid(x)
        else:
            p = torch.nan_to_num(torch.softmax(x, 1))
        rank = p.clone() if s["bias"] is None else p + s["bias"].double()
        rank[off] = -1e300
        if groups > 1:
            inside = rank.unflatten(1, (groups, -1))
            top = inside.topk(case["group_top"], dim=2)[0]
            strength = top.masked_fill(top < -1e299, 0.0).sum(2).masked_fill(top[:, :, 0] < -1e299, -1e300)
            cut = strength.topk(case["top_groups"], dim=1)[0][:, -1:]
            rank = inside.masked_fill((strength < cut)[:, :, None], -1e300).flatten(1)
        # stable order: the index breaks ties
        at = torch.argsort(rank, dim=1, descending=True, stable=True)[:, :k]
        on = rank.gather(1, at) > -1e299
        q = p.gather(1, at) * on
        total = q.sum(1, keepdim=True) + 1e-20
        weights.append(q / total if case["renorm"] else q)
        if case["grad"]:
            up = s["d_weight"][lo:lo + 131072].double() * on
            dq = (up / total - (up * q).sum(1, keepdim=True) / total ** 2) * on if case["renorm"] else up
            dp = torch.zeros_like(p).scatter_add(1, at, dq)
            local = p * (1 - p) * dp if case["score"] == "sigmoid" else p * dp - p * (p * dp).sum(1, keepdim=True)
            slopes.append(local)
    out = dict(expert=None, weight=torch.cat(weights), offsets=None, row_token=None, token_row=None)
    if case["grad"]:
        out["d_logits"] = torch.cat(slopes)
    return out


def _exact_product(case, s):
    z = torch.empty(s["out"].shape, dtype=torch.float64, device=_DEV)
    for e in range(case["experts"]):
        rows = slice(s["bounds"][e], s["bounds"][e + 1])
        x = s["x"][s["row_token"][rows].long()] if case["gather"] else s["x"][rows]
        z[rows] = torch.addmm(s["bias"][e].double(), x.double(), s["w"][e].double().T)
    return z.clamp_min(0.0) if case["relu"] else z


def _exact_product_grad(case, s):
    out = dict(dw=torch.zeros(s["dw"].shape, dtype=torch.float64, device=_DEV),
               db=torch.zeros(s["db"].shape, dtype=torch.float64, device=_DEV))
    if case["dx"]:
        out["dx"] = torch.zeros(s["dx"].shape, dtype=torch.float64, device=_DEV)
    for e in range(case["experts"]):
        rows = slice(s["bounds"][e], s["bounds"][e + 1])
        x = (s["x"][s["row_token"][rows].long()] if case["gather"] else s["x"][rows]).double()
        up = s["dz"][rows].double()
        out["dw"][e] = torch.mm(up.T, x)
        out["db"][e] = up.sum(0)
        if case["dx"]:
            down = torch.mm(up, s["w"][e].double())
            out["dx"][rows] = down * (x > 0) if case["relu"] else down
    return out


def _exact_combine(case, s):
    n, k, f = case["tokens"], case["top_k"], case["features"]
    weight = s["weight"].double()
    if not case["grad"]:
        out = torch.zeros(n, f, dtype=torch.float64, device=_DEV)
        for j in range(k):
            out += weight[:, j:j + 1] * s["y"][s["token_row"][:, j].long()].double()
        return out
    dy = torch.zeros(n * k, f, dtype=torch.float64, device=_DEV)
    d_weight = torch.zeros(n, k, dtype=torch.float64, device=_DEV)
    up = s["d_out"].double()
    for j in range(k):
        at = s["token_row"][:, j].long()
        dy[at] = weight[:, j:j + 1] * up
        d_weight[:, j] = torch.einsum("nf,nf->n", s["y"][at].double(), up)
    return dict(dy=dy, d_weight=d_weight)


def _exact_clip(case, s):
    square = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    norm = math.sqrt(square)
    factor = min(1.0, case["norm"] / (norm + 1e-6))
    return dict(norm=torch.tensor([norm], dtype=torch.float64), grads=[g.double() * factor for g in s["grads"]])


def exact(case, seed):
    s = prepare(case, seed)
    return dict(route=_exact_route, product=_exact_product, product_grad=_exact_product_grad,
                combine=_exact_combine, clip=_exact_clip)[case["op"]](case, s)
