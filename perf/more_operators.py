"""What is measured of the length predictor's encoder: the lookup of its tokens' embeddings, the gated
recurrence over a request's window, dropout with a residual, dense layers with bias, activation and
residual, each with its gradient.

``own`` false: the plain form, elementary torch operations in 32 bits.  ``own`` true: the calls a
user makes of the library.  ``prepare`` makes inputs and the output buffers that a program keeps.
"""
import functools
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_DEV = "cuda"


def listed():
    return [
        # a quiet scheduling tick: the newest tokens of a few requests are looked up (latency)
        dict(name="embed 300 x 256", op="embed", tokens=300, vocabulary=8192, features=256, type="f32", grad=False),
        # the token windows of a training batch, scaled
        dict(name="embed 524288 x 1024", op="embed", tokens=524288, vocabulary=131072, features=1024, type="bf16", grad=False),
        # ... and the gradient of the table: few tokens are frequent, many are rare, some occur nowhere
        dict(name="embed grad 524288 x 1024", op="embed", tokens=524288, vocabulary=131072, features=1024, type="bf16", grad=True),
        # re-prediction of running requests: every request's state takes one more token, in place
        dict(name="recurrence step 4096 x 1024", op="recurrence", sequences=4096, longest=1, ragged=False, features=1024,
             type="bf16", grad=False, missing=False),
        # a few long histories with missing observations
        dict(name="recurrence 4 x 32768 x 1024", op="recurrence", sequences=4, longest=32768, ragged=False, features=1024,
             type="bf16", grad=False, missing=True),
        # training over windows of unequal length, forward and backward, odd width
        dict(name="recurrence 500 x 512 ragged x 520 + grad", op="recurrence", sequences=500, longest=512, ragged=True,
             features=520, type="bf16", grad=True, missing=True),
        # a small batch's states, odd sizes, 32 bits (latency)
        dict(name="dropout 333 x 250", op="dropout", rows=333, features=250, p=0.1, residual=False, type="f32"),
        # a training batch's block: dropped, scaled and added to what went around it
        dict(name="dropout 131072 x 1024 residual", op="dropout", rows=131072, features=1024, p=0.1, residual=True, type="bf16"),
        # a handful of running requests through a layer (latency: the weights' read)
        dict(name="linear 5 x 2048 to 1024", op="linear", rows=5, fan_in=2048, fan_out=1024, activation="silu", bias=True,
             residual=False, keep=False, type="bf16"),
        # odd sizes, a middling batch, 16-bit floats
        dict(name="linear 1003 x 1000 to 504 residual", op="linear", rows=1003, fan_in=1000, fan_out=504, activation="relu",
             bias=True, residual=True, keep=False, type="f16"),
        # a block's second layer in training: activation, residual, the sums kept for the gradient
        dict(name="linear 65536 x 2048 to 2048 residual", op="linear", rows=65536, fan_in=2048, fan_out=2048,
             activation="gelu", bias=True, residual=True, keep=True, type="bf16"),
        # the gradient of a block's first layer, its input the activation of the layer below, which the block also passes on
        dict(name="linear grad 16384 x 2048 to 1024", op="linear_grad", rows=16384, fan_in=2048, fan_out=1024,
             activation="gelu", bias=True, around=True, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["embed", "embed", "recurrence", "recurrence", "recurrence", "dropout", "linear", "linear", "linear_grad"])
    if op == "embed":
        features = _log_int(rng, 8, 2048)
        vocabulary = _log_int(rng, 500, min(262144, 134217728 // features))
        return dict(op=op, tokens=_log_int(rng, 100, min(1048576, 536870912 // features)), vocabulary=vocabulary, features=features,
                    type=rng.choice(["f32", "bf16", "f16"]), grad=rng.random() < 0.6)
    if op == "recurrence":
        features = _log_int(rng, 16, 2048)
        sequences = _log_int(rng, 1, 8192)
        longest = _log_int(rng, 1, max(2, min(32768, 100000000 // (features * sequences))))
        return dict(op=op, sequences=sequences, longest=longest, ragged=longest > 1 and rng.random() < 0.6, features=features,
                    type=rng.choice(["f32", "bf16", "f16"]), grad=rng.random() < 0.5, missing=rng.random() < 0.5)
    if op == "dropout":
        features = _log_int(rng, 8, 4096)
        return dict(op=op, rows=_log_int(rng, 100, 100000000 // features), features=features, p=round(rng.uniform(0.02, 0.6), 3),
                    residual=rng.random() < 0.5, type=rng.choice(["f32", "bf16", "f16"]))
    fan_in, fan_out = _log_int(rng, 32, 4096), _log_int(rng, 32, 4096)
    if rng.random() < 0.1:
        fan_out = 1                                  # the answer itself
    per_row = 2.0 * fan_in * fan_out * (2 if op == "linear_grad" else 1)
    rows = _log_int(rng, 1 if op == "linear" else 64, int(max(65, min(65536, 4.0e11 / per_row))))
    case = dict(op=op, rows=rows, fan_in=fan_in, fan_out=fan_out, activation=rng.choice(["none", "relu", "gelu", "silu"]),
                bias=rng.random() < 0.8, type=rng.choice(["bf16", "f16"]))
    if op == "linear":
        case.update(residual=rng.random() < 0.5, keep=rng.random() < 0.4)
    else:
        case["around"] = rng.random() < 0.5
    return case


# ---- inputs ---------------------------------------------------------------------------------

def _generator(case, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _padded(rows, cols, dtype):
    """Rows that start 16-byte aligned, as the library wants them: [rows, cols] of a wider buffer."""
    ld = (cols + 7) // 8 * 8
    return torch.zeros(rows, ld, dtype=dtype, device=_DEV)[:, :cols]


def _normal(rows, cols, dtype, g, scale=1.0):
    out = _padded(rows, cols, dtype)
    out.copy_(torch.randn(rows, cols, generator=g, device=_DEV) * scale)
    return out


def _tokens(n, vocabulary, g):
    """Token numbers as text has them: the r-th most frequent about 1 / r as often; one in two hundred is padding."""
    u = torch.rand(n, generator=g, device=_DEV, dtype=torch.float64)
    rank = torch.exp(u * math.log(vocabulary + 1)).long().sub_(1).clamp_(0, vocabulary - 1)
    ids = torch.randperm(vocabulary, generator=g, device=_DEV)[rank].to(torch.int32)
    ids[torch.rand(n, generator=g, device=_DEV) < 0.005] = -1
    return ids


def _prepare_embed(case, g):
    n, v, f, t = case["tokens"], case["vocabulary"], case["features"], _TYPES[case["type"]]
    s = dict(ids=_tokens(n, v, g), scale=math.sqrt(f))
    if case["grad"]:
        s["d_out"] = _normal(n, f, t, g, 0.05)
        s["d_table"] = _padded(v, f, torch.float32)
    else:
        s["table"] = _normal(v, f, t, g, f ** -0.5)
        s["out"] = _padded(n, f, t)
    return s


def _lengths(case, g):
    """Lengths of the sequences: all the same, or spread from few rows (none, where there are many) to the longest."""
    n, longest = case["sequences"], case["longest"]
    if not case["ragged"]:
        return [longest] * n
    spread = [longest * (j + 1) // n for j in range(n)]
    return [spread[j] for j in torch.randperm(n, generator=g, device=_DEV).tolist()]


def _prepare_recurrence(case, g):
    f, n, t = case["features"], case["sequences"], _TYPES[case["type"]]
    lengths = _lengths(case, g)
    rows = sum(lengths)
    offsets = torch.zeros(n + 1, dtype=torch.int64)
    offsets[1:] = torch.tensor(lengths).cumsum(0)
    s = dict(lengths=lengths, bounds=offsets.to(_DEV), offsets=offsets.to(torch.int32).to(_DEV))
    s["x"] = _normal(rows, f, t, g)
    s["gate"] = _normal(rows, f, t, g, 1.5)
    s["gate"].add_(2.0)                               # most of the state stays
    if case["missing"]:                               # nothing observed: the state stays as it is
        s["gate"][torch.rand(rows, generator=g, device=_DEV) < 0.02] = math.inf
    s["h0"] = _normal(n, f, torch.float32, g, 0.5)
    s["out"], s["last"] = _padded(rows, f, t), _padded(n, f, torch.float32)
    if case["grad"]:
        s["d_out"], s["d_last"] = _normal(rows, f, t, g, 0.05), _normal(n, f, torch.float32, g, 0.05)
        s["dx"], s["d_gate"], s["d_h0"] = _padded(rows, f, t), _padded(rows, f, t), _padded(n, f, torch.float32)
        if own:
            s["states"] = _library().gated_scan_states(rows, n, f)
    return s


def _prepare_dropout(case, g):
    r, f, t = case["rows"], case["features"], _TYPES[case["type"]]
    s = dict(x=_normal(r, f, t, g), out=_padded(r, f, t),
             rng=torch.randint(0, 2 ** 62, (2,), generator=g, device=_DEV, dtype=torch.int64))      # seed and place in the stream
    s["residual"] = _normal(r, f, t, g) if case["residual"] else None
    return s


def _prepare_linear(case, g):
    r, i, o, t = case["rows"], case["fan_in"], case["fan_out"], _TYPES[case["type"]]
    return dict(x=_normal(r, i, t, g), w=_normal(o, i, t, g, 1.5 * i ** -0.5),
                bias=torch.randn(o, generator=g, device=_DEV) * 0.2 if case["bias"] else None,
                residual=_normal(r, o, t, g) if case["residual"] else None,
                z=_padded(r, o, t) if case["keep"] else None, out=_padded(r, o, t))


def _prepare_linear_grad(case, g):
    r, i, o, t = case["rows"], case["fan_in"], case["fan_out"], _TYPES[case["type"]]
    s = dict(x=_normal(r, i, t, g), w=_normal(o, i, t, g, i ** -0.5), dz=_normal(r, o, t, g, 0.05))
    active = case["activation"] != "none"
    s["z_below"] = _normal(r, i, t, g, 1.2) if active else None      # what the layer below kept, its activation is x
    if active:
        s["x"].copy_(_activate(s["z_below"].float(), case["activation"]))
    s["around"] = _normal(r, i, t, g, 0.05) if case["around"] else None
    s["dz_below"] = _padded(r, i, t) if active else None
    s["dx"] = _padded(r, i, t) if case["around"] or not active else None
    s["dw"] = _padded(o, i, torch.float32)
    s["db"] = torch.empty(o, device=_DEV) if case["bias"] else None
    return s


def prepare(case, seed):
    g = _generator(case, seed)
    s = dict(embed=_prepare_embed, recurrence=_prepare_recurrence, dropout=_prepare_dropout, linear=_prepare_linear,
             linear_grad=_prepare_linear_grad)[case["op"]](case, g)
    s["case"] = case
    return s


# ---- plain forms ----------------------------------------------------------------------------

def _plain_embed(s):
    ids = s["ids"].long()
    there = (ids >= 0)[:, None]
    if not s["case"]["grad"]:
        rows = s["table"][ids.clamp_min(0)].float() * s["scale"]
        return torch.where(there, rows, 0.0).to(s["table"].dtype)
    up = torch.where(there, s["d_out"].float() * s["scale"], 0.0)
    return torch.zeros(s["d_table"].shape, dtype=torch.float32, device=_DEV).index_add_(0, ids.clamp_min(0), up)


def _scan(a, b, longest):
    """h[t] = a[t] h[t - 1] + b[t] down the rows, by doubling; a sequence begins with a = 0."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _plain_recurrence(s):
    case, bounds = s["case"], s["bounds"]
    some = bounds[1:] > bounds[:-1]                   # sequences with a row
    first, last = bounds[:-1][some], bounds[1:][some] - 1
    x, g = s["x"].float(), s["gate"].float()
    a, c = 1.0 / (1.0 + torch.exp(-g)), 1.0 / (1.0 + torch.exp(g))
    keep, b = a.clone(), c * x
    b[first] += a[first] * s["h0"][some]
    keep[first] = 0.0
    h = _scan(keep, b, case["longest"])
    end = s["h0"].clone()
    end[some] = h[last]
    out = dict(out=h.to(s["x"].dtype), last=end)
    if case["grad"]:
        before = torch.cat([h[:1], h[:-1]])
        before[first] = s["h0"][some]
        up = s["d_out"].to(torch.float32, copy=True)
        up[last] += s["d_last"][some]
        back = torch.cat([a[1:], a[:1]])
        back[last] = 0.0
        up = _scan(back.flip(0), up.flip(0), case["longest"]).flip(0)
        d_h0 = s["d_last"].clone()
        d_h0[some] = a[first] * up[first]
        out.update(dx=(c * up).to(s["x"].dtype), d_gate=(a * c * (before - x) * up).to(s["x"].dtype), d_h0=d_h0)
    return out


_LOW = 0xFFFFFFFF


def _halves(n, rng):
    """Philox-4x32 with ten rounds: the first n of the 16-bit halves (eight a counter) for the counters 0, 1, ... of a stream."""
    seed, place = rng[0], rng[1]
    count = torch.arange((n + 7) // 8, device=_DEV)
    c = [count & _LOW, count >> 32, (place & _LOW).expand_as(count), ((place >> 32) & _LOW).expand_as(count)]
    k = [seed & _LOW, (seed >> 32) & _LOW]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # (the products wrap; their 64 bits are the right ones)
        c = [((q >> 32) & _LOW) ^ c[1] ^ k[0], q & _LOW, ((p >> 32) & _LOW) ^ c[3] ^ k[1], p & _LOW]
        k = [(k[0] + 0x9E3779B9) & _LOW, (k[1] + 0xBB67AE85) & _LOW]
    return torch.stack([half for word in c for half in (word & 0xFFFF, word >> 16)], 1).view(-1)[:n]


def _plain_dropout(s):
    x, out_of = s["x"].float(), round(s["case"]["p"] * 65536.0)      # p in steps of 2^-16
    kept = _halves(x.numel(), s["rng"]).view(x.shape) >= out_of
    y = torch.where(kept, x * (65536.0 / (65536.0 - out_of)), 0.0)
    return (y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype)


_GELU_IN, _GELU_CUBE = math.sqrt(2.0 / math.pi), 0.044715


def _activate(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return z / (1.0 + torch.exp(-2.0 * _GELU_IN * (z + _GELU_CUBE * z * z * z)))
    return z


def _slope(z, name):
    if name == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s + z * s * (1.0 / (1.0 + torch.exp(z)))
    u = 2.0 * _GELU_IN * (z + _GELU_CUBE * z * z * z)
    s, rest = 1.0 / (1.0 + torch.exp(-u)), 1.0 / (1.0 + torch.exp(u))
    return s + z * s * rest * (2.0 * _GELU_IN * (1.0 + 3.0 * _GELU_CUBE * z * z))


def _plain_linear(s):
    case, t = s["case"], s["x"].dtype
    z = s["x"].float() @ s["w"].float().T
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _activate(z, case["activation"])
    out = dict(out=(y if s["residual"] is None else y + s["residual"].float()).to(t))
    if case["keep"]:
        out["z"] = z.to(t)
    return out


def _plain_linear_grad(s):
    case, dz = s["case"], s["dz"].float()
    dx = dz @ s["w"].float()
    if s["around"] is not None:
        dx = dx + s["around"].float()
    out = dict(dw=dz.T @ s["x"].float())
    if s["dx"] is not None:
        out["dx"] = dx.to(s["x"].dtype)
    if s["dz_below"] is not None:
        out["dz_below"] = (dx * _slope(s["z_below"].float(), case["activation"])).to(s["x"].dtype)
    if case["bias"]:
        out["db"] = dz.sum(0)
    return out


# ---- the library's operators ----------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _library():
    import paper_2605_16867_b200 as lib
    return lib.GoodServe(torch.cuda.current_device())


def _own_embed(s):
    gs = _library()
    if s["case"]["grad"]:
        gs.embedding_backward(s["d_out"], s["ids"], s["d_table"], scale=s["scale"])
        return s["d_table"]
    gs.embedding(s["table"], s["ids"], s["out"], scale=s["scale"])
    return s["out"]


def _own_recurrence(s):
    gs, out = _library(), dict(out=s["out"], last=s["last"])
    if not s["case"]["grad"]:
        gs.gated_scan(s["x"], s["gate"], s["offsets"], out=s["out"], h0=s["h0"], last=s["last"])
        return out
    gs.gated_scan(s["x"], s["gate"], s["offsets"], out=s["out"], h0=s["h0"], last=s["last"], states=s["states"])
    gs.gated_scan_backward(s["x"], s["gate"], s["offsets"], s["states"], s["dx"], s["d_gate"], d_out=s["d_out"],
                           d_last=s["d_last"], d_h0=s["d_h0"])
    return dict(out, dx=s["dx"], d_gate=s["d_gate"], d_h0=s["d_h0"])


def _own_dropout(s):
    _library().dropout(s["x"], s["rng"], s["case"]["p"], s["out"], residual=s["residual"])
    return s["out"]


def _own_linear(s):
    _library().linear(s["x"], s["w"], s["out"], bias=s["bias"], activation=s["case"]["activation"], residual=s["residual"],
                      z=s["z"])
    return dict(out=s["out"], z=s["z"]) if s["case"]["keep"] else dict(out=s["out"])


def _own_linear_grad(s):
    _library().linear_backward(s["dz"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], db=s["db"], around=s["around"],
                               z_below=s["z_below"], activation=s["case"]["activation"], dz_below=s["dz_below"])
    return {k: s[k] for k in ("dx", "dz_below", "dw", "db") if s[k] is not None}


_PLAIN = dict(embed=_plain_embed, recurrence=_plain_recurrence, dropout=_plain_dropout, linear=_plain_linear,
              linear_grad=_plain_linear_grad)
_OWN = dict(embed=_own_embed, recurrence=_own_recurrence, dropout=_own_dropout, linear=_own_linear, linear_grad=_own_linear_grad)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    op, width = case["op"], {"f32": 4, "bf16": 2, "f16": 2}[case["type"]]
    if op == "embed":
        n, v, f = case["tokens"], case["vocabulary"], case["features"]
        if case["grad"]:
            return dict(bytes=4 * n + n * f * width + 4 * v * f, flops=1.0 * n * f)
        # distinct tokens among n whose r-th most frequent has probability 1 / (r ln v): about
        probability = 1.0 / math.log(v + 1)
        distinct = sum(1.0 - math.exp(-n * probability / r) for r in range(1, min(v, 2000) + 1))
        if v > 2000:                                  # the rest by strips of equal logarithm
            edges = [2000.0 * (v / 2000.0) ** (j / 64.0) for j in range(65)]
            distinct += sum((b - a) * (1.0 - math.exp(-n * probability / math.sqrt(a * b))) for a, b in zip(edges, edges[1:]))
        return dict(bytes=int(4 * n + n * f * width + distinct * f * width), flops=1.0 * n * f)
    if op == "recurrence":
        n, f = case["sequences"], case["features"]
        rows = sum(case["longest"] * (j + 1) // n for j in range(n)) if case["ragged"] else n * case["longest"]
        passes = 3 if not case["grad"] else 6         # x, gate and out; with the gradient also d_out, dx and d_gate
        size = rows * f * width * passes + n * f * 4 * (2 if not case["grad"] else 4) + 4 * (n + 1)
        return dict(bytes=int(size), flops=rows * f * (10.0 if not case["grad"] else 30.0))
    if op == "dropout":
        n = case["rows"] * case["features"]
        return dict(bytes=n * width * (3 if case["residual"] else 2) + 16, flops=2.0 * n)
    r, i, o = case["rows"], case["fan_in"], case["fan_out"]
    if op == "linear":
        size = (r * i + o * i + r * o * (1 + (1 if case["residual"] else 0) + (1 if case["keep"] else 0))) * width
        return dict(bytes=size + (4 * o if case["bias"] else 0), flops=2.0 * r * i * o)
    active = case["activation"] != "none"             # then z_below is read and dz_below written
    size = (r * o + r * i * (1 + 2 * active + case["around"] + (case["around"] or not active)) + o * i) * width
    return dict(bytes=size + 4 * o * i + (4 * o if case["bias"] else 0), flops=4.0 * r * i * o)


# ---- the definitions in 64 bits -------------------------------------------------------------

def _exact_embed(case, s):
    ids = s["ids"]
    if not case["grad"]:
        out = torch.zeros(len(ids), case["features"], dtype=torch.float64, device=_DEV)
        real = (ids != -1).nonzero()[:, 0]
        for part in real.split(65536):
            out[part] = s["table"].index_select(0, ids[part]).double().mul_(s["scale"])
        return out
    # the rows of a token lie together after sorting: differences of running sums would lose digits, so rounds of pairs
    order = torch.argsort(ids.long(), stable=True)
    order = order[int((ids < 0).sum()):]
    key = ids.long()[order]
    out = torch.zeros(case["vocabulary"], case["features"], dtype=torch.float64, device=_DEV)
    for columns in torch.arange(case["features"], device=_DEV).split(64):
        value, token = s["d_out"][:, columns].double()[order], key
        while len(token) and bool((token[1:] == token[:-1]).any()):
            fresh = torch.ones(len(token), dtype=torch.bool, device=_DEV)
            fresh[1:] = token[1:] != token[:-1]
            start = torch.where(fresh, torch.arange(len(token), device=_DEV), 0).cummax(0)[0]
            even = (torch.arange(len(token), device=_DEV) - start) % 2 == 0
            value = value.clone()
            at = (~even).nonzero()[:, 0]
            value[at - 1] += value[at]
            value, token = value[even], token[even]
        out[token[:, None], columns[None, :]] = value * s["scale"]
    return out


def _stacked(s, name, fill=0.0):
    """The rows of the sequences side by side: [longest, sequences, features] in 64 bits."""
    lengths = torch.tensor(s["lengths"], device=_DEV)
    longest = max(1, int(lengths.max()))
    t = torch.arange(longest, device=_DEV)[:, None]
    there = t < lengths[None, :]
    full = torch.full((longest, len(lengths), s[name].shape[1]), fill, dtype=torch.float64, device=_DEV)
    full[there] = s[name].double()[(s["bounds"][:-1][None, :] + t)[there]]
    return full, there


def _exact_recurrence(case, s):
    if case["longest"] * case["sequences"] * case["features"] > 140000000:
        return None
    gate, there = _stacked(s, "gate", math.inf)
    x = _stacked(s, "x")[0]
    a = torch.sigmoid(gate)
    c = torch.sigmoid(-gate)
    del gate
    h = s["h0"].double()
    states = torch.empty_like(x)
    for t in range(len(x)):
        h = torch.addcmul(c[t] * x[t], a[t], h)
        states[t] = h
    flat = (s["bounds"][:-1][None, :] + torch.arange(len(x), device=_DEV)[:, None])[there]

    def packed(values):
        out = torch.empty(s["x"].shape, dtype=torch.float64, device=_DEV)
        out[flat] = values[there]
        return out
    out = dict(out=packed(states), last=h)
    if case["grad"]:
        up = _stacked(s, "d_out")[0]
        d = s["d_last"].double()
        dx, d_gate = torch.empty_like(x), torch.empty_like(x)
        for t in reversed(range(len(x))):
            d = d + up[t]
            before = states[t - 1] if t else s["h0"].double()
            dx[t] = d * c[t]
            d_gate[t] = d * (before - x[t]) * (a[t] * c[t])
            d = d * a[t]
        out.update(dx=packed(dx), d_gate=packed(d_gate), d_h0=d)
    return out


def _exact_dropout(case, s):
    """Each row by itself; the products in 16-bit halves."""
    seed, place = (int(v) for v in s["rng"].tolist())
    out = torch.empty(s["x"].shape, dtype=torch.float64, device=_DEV)
    f = case["features"]

    def high(v, m):
        return (m * (v >> 16) + ((m * (v & 0xFFFF)) >> 16)) >> 16

    def low(v, m):
        return ((((m * (v >> 16)) & 0xFFFF) << 16) + m * (v & 0xFFFF)) & _LOW
    for rows in torch.arange(len(out), device=_DEV).split(max(1, 33554432 // f)):
        index = rows[:, None] * f + torch.arange(f, device=_DEV)[None, :]
        x0, x1 = (index // 8) % 2 ** 32, (index // 8) // 2 ** 32
        x2, x3 = torch.full_like(index, place % 2 ** 32), torch.full_like(index, place // 2 ** 32 % 2 ** 32)
        k0, k1 = seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32
        for j in range(10):
            x0, x1, x2, x3 = (high(x2, 0xCD9E8D57) ^ x1 ^ ((k0 + j * 0x9E3779B9) % 2 ** 32), low(x2, 0xCD9E8D57),
                              high(x0, 0xD2511F53) ^ x3 ^ ((k1 + j * 0xBB67AE85) % 2 ** 32), low(x0, 0xD2511F53))
        pick = index % 8 // 2
        word = torch.where(pick == 0, x0, torch.where(pick == 1, x1, torch.where(pick == 2, x2, x3)))
        half = torch.where(index % 2 == 0, word % 65536, word // 65536).double()
        cut = round(case["p"] * 65536.0)
        out[rows] = s["x"][rows].double() / (1.0 - cut / 65536.0) * (half > cut - 0.5)
    return out if s["residual"] is None else out + s["residual"].double()


def _exact_activation(z, name):
    if name == "relu":
        return z.clamp_min(0.0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(_GELU_IN * (z + _GELU_CUBE * z ** 3)))
    return z


def _exact_linear(case, s):
    z = torch.mm(s["x"].double(), s["w"].double().T)
    if s["bias"] is not None:
        z += s["bias"].double()
    y = _exact_activation(z, case["activation"])
    out = dict(out=y if s["residual"] is None else s["residual"].double() + y)
    if case["keep"]:
        out["z"] = z
    return out


def _exact_linear_grad(case, s):
    dz = s["dz"].double()
    dx = torch.mm(dz, s["w"].double())
    if s["around"] is not None:
        dx += s["around"].double()
    out = dict(dw=torch.mm(dz.T, s["x"].double()))
    if s["dx"] is not None:
        out["dx"] = dx
    if s["dz_below"] is not None:
        with torch.enable_grad():                     # the slope by differentiation
            z = s["z_below"].double().requires_grad_()
            out["dz_below"] = torch.autograd.grad(_exact_activation(z, case["activation"]), z, dx)[0]
    if case["bias"]:
        out["db"] = torch.einsum("ro->o", dz)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return dict(embed=_exact_embed, recurrence=_exact_recurrence, dropout=_exact_dropout, linear=_exact_linear,
                linear_grad=_exact_linear_grad)[case["op"]](case, s)
