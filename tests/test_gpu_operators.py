"""The length predictor's operators (expert routing, the experts' products, their combination,
gradient clipping) against plain implementations in 64 bits.

Tolerances, fixed before the first run.  u is the unit roundoff of the output's type (2^-24, 2^-8 for
bfloat16, 2^-11 for float16).  A dot product of n terms in float is off by at most (n + 8) * 2^-23 times the
sum of the terms' magnitudes (2^-23: the tensor cores may truncate), then rounded once to the output: u * |value|.
Scores pass through one exponential, one division and up to 32 partial sums: 2^-19 relative; a weight's or a
logit's gradient is a sum of at most top_k + 2 such products: 2^-17 times the sum of their magnitudes."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
BAD_VALUE = 4


@pytest.fixture(scope="module")
def gs():
    from paper_2605_16867_b200 import GoodServe
    assert torch.cuda.is_available()
    g = GoodServe(0)
    yield g
    g.close()


@pytest.fixture(autouse=True)
def clean_status(gs):
    gs.device_status()
    yield


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def padded(rows, cols, dtype, fill=float("nan"), extra=0):
    """A matrix inside a wider buffer whose other columns hold NaN."""
    ld = (cols + 7) // 8 * 8 + 8 * extra
    return torch.full((rows, ld), fill, dtype=dtype, device="cuda")[:, :cols]


def rest(t):
    """What lies between the rows of a padded matrix."""
    return torch.as_strided(t, (t.shape[0], t.stride(0) - t.shape[1]), (t.stride(0), 1), t.storage_offset() + t.shape[1])


def normal(rows, cols, dtype, g, scale=1.0, extra=0):
    t = padded(rows, cols, dtype, extra=extra)
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return t


def close(got, want, room):
    err = (got.double() - want).abs()
    bad = ~(err <= room)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off; worst {float((err / room.clamp_min(1e-300)).max()):.3g} x the bound"


# ---- routing ----------------------------------------------------------------------------------

def reference_route(x, bias, k, score, groups, top_groups, group_top, renormalise, scale):
    """Definition in 64 bits.  Also: how far the last bits of a score are from deciding each row."""
    x = x.double().clamp_max(3.4028234663852886e38)
    on = ~(torch.isnan(x) | (x == -math.inf))
    if bias is not None:
        on = on & (bias != -math.inf)
    xs = torch.where(torch.isnan(x), -math.inf, x)
    if score == "sigmoid":
        s = torch.where(xs == -math.inf, 0.0, torch.sigmoid(xs))
    else:
        s = torch.nan_to_num(torch.softmax(xs, 1))
    c = s if bias is None else s + bias.double()
    c = torch.where(on, c, -math.inf)
    margin = torch.full((len(c),), math.inf, dtype=torch.float64, device=x.device)

    def gaps(v):
        d = v[:, :-1] - v[:, 1:]
        d = torch.where((d == 0) | torch.isnan(d), math.inf, d)
        return d.amin(1) if d.shape[1] else torch.full((len(v),), math.inf, dtype=torch.float64, device=v.device)
    if groups > 1:
        parts = c.view(len(c), groups, -1)
        best = parts.sort(2, descending=True)[0][:, :, :group_top]
        g = torch.where(best[:, :, 0] == -math.inf, -math.inf, torch.where(best == -math.inf, 0.0, best).sum(2))
        v, at = torch.sort(g, dim=1, descending=True, stable=True)
        margin = torch.minimum(margin, gaps(v))
        keep = torch.zeros_like(g, dtype=torch.bool).scatter_(1, at[:, :top_groups], True)
        c = torch.where(keep[:, :, None], parts, -math.inf).view_as(c)
    v, at = torch.sort(c, dim=1, descending=True, stable=True)
    margin = torch.minimum(margin, gaps(v[:, :k + 1]))
    there = v[:, :k] > -math.inf
    expert = torch.where(there, at[:, :k], -1)
    q = torch.where(there, s.gather(1, at[:, :k]), 0.0)
    w = scale * (q / (q.sum(1, keepdim=True) + 1e-20) if renormalise else q)
    return s, expert, w, margin


def reference_order(expert, n_experts):
    n, k = expert.shape
    flat = expert.reshape(-1).cpu().numpy()
    order = np.argsort(np.where(flat < 0, n_experts, flat), kind="stable")
    order = order[: int((flat >= 0).sum())]
    offsets = np.zeros(n_experts + 1, np.int64)
    offsets[1:] = np.cumsum(np.bincount(flat[flat >= 0], minlength=n_experts))
    row_token = np.full(n * k, -1)
    row_token[: len(order)] = order // k
    token_row = np.full(n * k, -1)
    token_row[order] = np.arange(len(order))
    return offsets, row_token, token_row.reshape(n, k)


def route(gs, x, router, bias=None):
    n, k, e = x.shape[0], router.top_k, router.n_experts
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [torch.full((n, k), -9, **i32), torch.full((n, k), -9.0, device="cuda"), torch.full((e + 1,), -9, **i32),
           torch.full((n * k,), -9, **i32), torch.full((n, k), -9, **i32)]
    gs.expert_route(x, router, *out, bias=bias)
    return out


def check_route(gs, x, router, bias, spec):
    expert, weight, offsets, row_token, token_row = route(gs, x, router, bias)
    s, ref, w, margin = reference_route(x, bias, *spec)
    clear = margin > 2e-6
    assert clear.float().mean() > 0.97 or len(x) < 40
    assert torch.equal(expert[clear].long(), ref[clear])
    # whatever the near ties went to, weights and order follow from the choice that was made
    there = expert >= 0
    q = torch.where(there, s.gather(1, expert.clamp_min(0).long()), 0.0)
    scale, renormalise = spec[-1], spec[-2]
    want = scale * (q / (q.sum(1, keepdim=True) + 1e-20) if renormalise else q)
    close(weight, want, 2.0 ** -19 * want.abs() + 1e-37)
    o, rt, tr = reference_order(expert, router.n_experts)
    assert np.array_equal(offsets.cpu().numpy(), o)
    assert np.array_equal(row_token.cpu().numpy(), rt)
    assert np.array_equal(token_row.cpu().numpy(), tr)
    # choices and weights alone: the same
    again = [torch.empty_like(expert), torch.empty_like(weight)]
    gs.expert_route(x, router, *again, bias=bias)
    assert torch.equal(again[0], expert) and torch.equal(again[1], weight)


ROUTERS = [
    # experts, top_k, score, groups, top_groups, group_top, renormalise, scale, bias
    (1, 1, "softmax", 1, 1, 1, True, 1.0, False),
    (2, 2, "sigmoid", 1, 1, 1, False, 2.5, False),
    (8, 3, "softmax", 2, 1, 2, True, 1.0, True),
    (9, 2, "softmax", 1, 1, 1, True, 1.0, False),
    (9, 9, "softmax", 1, 1, 1, True, 1.0, False),
    (16, 16, "softmax", 1, 1, 1, False, 1.0, True),
    (17, 5, "sigmoid", 1, 1, 1, True, 1.0, True),
    (32, 4, "softmax", 32, 9, 1, True, 1.0, True),
    (33, 4, "softmax", 1, 1, 1, True, 1.0, False),
    (60, 6, "sigmoid", 12, 5, 2, True, 1.0, True),
    (64, 8, "softmax", 8, 3, 1, True, 1.5, False),
    (100, 7, "sigmoid", 4, 2, 2, False, 1.0, True),
    (160, 6, "softmax", 8, 3, 2, False, 16.0, False),
    (256, 8, "sigmoid", 8, 4, 2, True, 2.5, True),
    (500, 10, "softmax", 1, 1, 1, True, 1.0, True),
    (512, 16, "sigmoid", 32, 7, 2, True, 1.0, True),
]


def make(spec):
    from paper_2605_16867_b200 import ExpertRouter
    e, k, score, groups, top_groups, group_top, ren, scale, _ = spec
    return ExpertRouter(e, k, score, groups, top_groups, group_top, ren, scale), (k, score, groups, top_groups, group_top, ren, scale)


@pytest.mark.parametrize("spec", ROUTERS, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}-g{s[3]}")
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_route(gs, spec, dtype):
    router, ref = make(spec)
    g = gen(spec[0] * 7 + 1)
    bias = torch.randn(spec[0], generator=g, device="cuda") * 0.1 if spec[-1] else None
    for n in (1, 31, 700):
        x = (torch.randn(n, spec[0], generator=g, device="cuda") * 2).to(dtype)
        check_route(gs, x, router, bias, ref)
    assert gs.device_status() == 0


@pytest.mark.parametrize("n", [0, 1, 2, 33, 1024, 1025, 5000, 70001])
def test_route_sizes(gs, n):
    for spec in (ROUTERS[3], ROUTERS[13]):
        router, ref = make(spec)
        g = gen(n + 5)
        bias = torch.randn(spec[0], generator=g, device="cuda") * 0.1 if spec[-1] else None
        x = torch.randn(n, spec[0], generator=g, device="cuda")
        if n:
            check_route(gs, x, router, bias, ref)
        else:
            assert route(gs, x, router, bias)[2].tolist() == [0] * (spec[0] + 1)


def test_route_ties_go_to_the_lowest_index(gs):
    for spec in (ROUTERS[3], ROUTERS[8], ROUTERS[10], ROUTERS[12]):
        router, ref = make(spec)
        x = torch.randint(0, 3, (3000, spec[0]), generator=gen(3), device="cuda").float() * 0.5
        check_route(gs, x, router, None, ref)
        expert = route(gs, torch.zeros(5, spec[0], device="cuda"), router)[0]
        if spec[3] == 1:
            assert expert.tolist() == [list(range(spec[1]))] * 5


def test_route_skewed_to_one_expert(gs):
    for spec in (ROUTERS[3], ROUTERS[13]):
        router, ref = make(spec)
        x = torch.randn(20000, spec[0], generator=gen(9), device="cuda")
        x[:, 3] += 8
        check_route(gs, x, router, None, ref)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_route_masks(gs, dtype):
    low = torch.finfo(dtype).min
    for spec in (ROUTERS[2], ROUTERS[3], ROUTERS[6], ROUTERS[9], ROUTERS[13]):
        router, ref = make(spec)
        e, g = spec[0], gen(11)
        x = (torch.randn(2000, e, generator=g, device="cuda") * 2).to(dtype)
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.5] = -math.inf
        x[:50] = -math.inf                                   # nothing left
        x[50:100, 1:] = -math.inf                            # one left
        x[100:200][torch.rand(100, e, generator=g, device="cuda") < 0.5] = low
        x[200:210] = low
        x[210:300, 2] = math.inf
        x[300:310] = math.inf
        if spec[3] > 1:
            x[400:500, : e // spec[3]] = -math.inf           # a group with nothing left
        check_route(gs, x, router, None, ref)
        bias = torch.zeros(e, device="cuda")
        bias[1] = -math.inf
        check_route(gs, x, router, bias, ref)
        assert gs.device_status() == 0
        expert, weight, _, _, _ = route(gs, x, router)
        assert (expert[:50] == -1).all() and (weight[:50] == 0).all()
        x[5:9] = math.nan
        x[600, 0] = math.nan
        check_route(gs, x, router, None, ref)
        assert gs.device_status() == BAD_VALUE


def test_route_strides(gs):
    router, ref = make(ROUTERS[3])
    for ld in (9, 11, 16):
        wide = torch.full((501, ld), math.nan, device="cuda")
        x = wide[:, :9]
        x.copy_(torch.randn(501, 9, generator=gen(ld), device="cuda"))
        check_route(gs, x, router, None, ref)
    assert gs.device_status() == 0


@pytest.mark.parametrize("spec", ROUTERS, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}-g{s[3]}")
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_route_backward(gs, spec, dtype):
    router, (k, score, groups, tg, gt, ren, scale) = make(spec)
    for n in (1, 333):
        g = gen(spec[0] + n)
        x = (torch.randn(n, spec[0], generator=g, device="cuda") * 2).to(dtype)
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.1] = -math.inf
        if n > 1:
            x[7] = -math.inf
        expert = route(gs, x, router)[0]
        dw = torch.randn(n, k, generator=g, device="cuda")
        wide = torch.full((n, spec[0] + 3), 7.0, dtype=dtype, device="cuda")
        out = wide[:, :spec[0]]
        gs.expert_route_backward(x, router, expert, dw, out)
        # the formula, by differentiation in 64 bits of the weights for this choice
        x64 = torch.where(x == -math.inf, -1e4, x.double()).requires_grad_()
        s = torch.sigmoid(x64) if score == "sigmoid" else torch.softmax(x64, 1)
        s = torch.where(x == -math.inf, 0.0, s)
        there = expert >= 0
        q = torch.where(there, s.gather(1, expert.clamp_min(0).long()), 0.0)
        t = q.sum(1, keepdim=True) + 1e-20
        w = scale * (q / t if ren else q)
        (w * dw.double()).sum().backward()
        want = torch.where((x == -math.inf), 0.0, x64.grad)
        dwd = dw.double().abs() * there
        room_q = scale * (dwd + (dwd * q / t).sum(1, keepdim=True)) / t if ren else scale * dwd
        room_q = torch.where(there, room_q, 0.0).detach()
        mag = torch.zeros_like(s).scatter_add_(1, expert.clamp_min(0).long(), room_q) * s.detach()
        if score == "softmax":
            mag = mag + s.detach() * (room_q * q.detach()).sum(1, keepdim=True)
        close(out, want, 2.0 ** -17 * mag + UNIT[dtype] * want.abs() + (2.0 ** -25 if dtype is F16 else 1e-37))
        assert (wide[:, spec[0]:] == 7).all()
    assert gs.device_status() == 0


def test_route_backward_against_differences(gs):
    for spec in (ROUTERS[3], ROUTERS[6], ROUTERS[9]):
        router, _ = make(spec)
        g = gen(77)
        x = torch.randn(40, spec[0], generator=g, device="cuda")
        expert = route(gs, x, router)[0]
        dw = torch.randn(40, spec[1], generator=g, device="cuda")
        out = torch.empty_like(x)
        gs.expert_route_backward(x, router, expert, dw, out)

        def loss(z):                                         # of the library's own forward, in slots of the same expert
            e2, w2 = route(gs, z, router)[:2]
            same = (e2 == expert).all(1)
            return (w2.double() * dw.double()).sum(1), same
        step = 1e-2
        for e in range(0, spec[0], 4):
            d = torch.zeros_like(x)
            d[:, e] = step
            (up, ok1), (down, ok2) = loss(x + d), loss(x - d)
            ok = ok1 & ok2
            assert ok.float().mean() > 0.5
            # central differences: step^2 / 6 times a third derivative of order one per unit of dw, and 2^-19 / step
            room = dw.double().abs().sum(1) * (step ** 2 + 2 * 2.0 ** -19 / step)
            assert ((out[:, e].double() - (up - down) / (2 * step)).abs() <= room)[ok].all()


def test_route_backward_ignores_experts_out_of_range(gs):
    router, _ = make(ROUTERS[3])
    x = torch.randn(10, 9, device="cuda")
    expert = torch.tensor([[0, 1]] * 10, dtype=torch.int32, device="cuda")
    clean = expert.clone()
    clean[4] = -1
    expert[4, 0], expert[4, 1] = 9, -7
    dw = torch.randn(10, 2, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    gs.expert_route_backward(x, router, clean, dw, a)
    assert gs.device_status() == 0
    gs.expert_route_backward(x, router, expert, dw, b)
    assert gs.device_status() == BAD_VALUE
    assert torch.equal(a, b)


# ---- products ---------------------------------------------------------------------------------

def layout(counts, g, tokens=None):
    """offsets of experts with these many rows, and a token for every row."""
    offsets = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    rows = int(offsets[-1])
    row_token = None if tokens is None else torch.randint(0, tokens, (rows,), generator=g, dtype=torch.int32, device="cuda")
    return offsets, rows, row_token


PRODUCTS = [
    # rows of each expert, in, out, gather
    ([1], 1, 1, False),
    ([0, 3, 0], 8, 8, False),
    ([5, 0, 1, 130], 64, 64, True),
    ([129, 64, 0, 255, 1], 65, 127, False),
    ([300, 17], 1000, 130, True),
    ([33] * 9, 512, 257, False),
    ([700, 1, 0, 90], 192, 1, True),
    ([1100], 320, 384, False),
    ([2, 3, 2, 1, 0, 4, 1, 1, 2], 2048, 1024, True),
    ([40, 3], 1, 300, True),
    ([1] * 200, 136, 72, False),
    ([64, 128, 256, 512], 128, 128, False),
    ([517, 0, 260], 263, 515, True),
]


def product_inputs(case, dtype, seed, extra=0):
    counts, i, o, gather = case
    g = gen(seed)
    offsets, rows, row_token = layout(counts, g, max(1, sum(counts) // 2) if gather else None)
    nx = max(1, sum(counts) // 2) if gather else rows
    x = normal(nx, i, dtype, g, extra=extra)
    w = padded(len(counts) * o, i, dtype, extra=extra)
    w.copy_(torch.randn(len(counts) * o, i, generator=g, device="cuda") * i ** -0.5)
    w = w.unflatten(0, (len(counts), o))
    bias = torch.randn(len(counts), o, generator=g, device="cuda")
    return g, offsets, rows, row_token, x, w, bias


def of_rows(x, row_token):
    return x if row_token is None else x[row_token.long()]


def segments(offsets):
    o = offsets.tolist()
    return [(e, slice(a, b)) for e, (a, b) in enumerate(zip(o[:-1], o[1:]))]


@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: f"{len(c[0])}e-{sum(c[0])}r-{c[1]}-{c[2]}")
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("relu", [False, True])
def test_linear(gs, case, dtype, relu):
    g, offsets, rows, row_token, x, w, bias = product_inputs(case, dtype, 5, extra=int(relu))
    b = bias if relu or case[2] % 2 else None
    spare = 3                                                # rows that no expert owns stay as they are
    out = padded(rows + spare, case[2], dtype, extra=int(relu))
    token = None if row_token is None else torch.cat([row_token, row_token.new_full((spare,), -1)])
    if row_token is None:
        x = torch.cat([x, x.new_full((spare, x.shape[1]), math.nan)]) if x.stride(0) == x.shape[1] else _with_rows(x, spare)
    gs.expert_linear(x, w, offsets, out, bias=b, row_token=token, relu=relu)
    xs = of_rows(x, row_token).double()
    for e, r in segments(offsets):
        z = xs[r] @ w[e].double().T
        mag = xs[r].abs() @ w[e].double().abs().T
        if b is not None:
            z, mag = z + b[e].double(), mag + b[e].double().abs()
        want = z.clamp_min(0) if relu else z
        close(out[r], want, (case[1] + 8) * 2.0 ** -23 * mag + UNIT[dtype] * want.abs() + 2.0 ** -25)
    assert torch.isnan(out[rows:]).all() and torch.isnan(rest(out)).all()
    assert gs.device_status() == 0


def _with_rows(x, spare):
    t = torch.full((x.shape[0] + spare, x.stride(0)), math.nan, dtype=x.dtype, device=x.device)[:, :x.shape[1]]
    t[: x.shape[0]] = x
    return t


@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: f"{len(c[0])}e-{sum(c[0])}r-{c[1]}-{c[2]}")
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("relu", [False, True])
def test_linear_backward(gs, case, dtype, relu):
    counts, i, o, _ = case
    g, offsets, rows, row_token, x, w, _ = product_inputs(case, dtype, 6, extra=int(relu))
    dz = normal(rows, o, dtype, g, extra=int(relu))
    dx = padded(rows, i, dtype, extra=int(relu))
    dw = torch.full((len(counts), o, (i + 3) // 4 * 4 + 4), math.nan, device="cuda")[..., :i]
    db = torch.full((len(counts), o), math.nan, device="cuda")
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx, dw=dw, db=db, row_token=row_token, relu_input=relu)
    xs, zs = of_rows(x, row_token).double(), dz.double()
    for e, r in segments(offsets):
        want = zs[r] @ w[e].double()
        mag = zs[r].abs() @ w[e].double().abs()
        if relu:
            want = torch.where(xs[r] > 0, want, 0.0)
        close(dx[r], want, (o + 8) * 2.0 ** -23 * mag + UNIT[dtype] * want.abs() + 2.0 ** -25)
        n = counts[e]
        close(dw[e], zs[r].T @ xs[r], (n + 8) * 2.0 ** -23 * (zs[r].abs().T @ xs[r].abs()) + 1e-30)
        close(db[e], zs[r].sum(0), (n + 8) * 2.0 ** -23 * zs[r].abs().sum(0) + 1e-30)
    assert torch.isnan(rest(dx)).all()
    # each output by itself: the same
    dx2, dw2 = padded(rows, i, dtype, extra=int(relu)), torch.empty_strided(dw.shape, dw.stride(), device="cuda")
    gs.expert_linear_backward(dz, x, w, offsets, dx=dx2, row_token=row_token, relu_input=relu)
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw2, row_token=row_token)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
    assert gs.device_status() == 0


def test_linear_gradients_against_differences(gs):
    g, offsets, rows, row_token, x, w, bias = product_inputs(([7, 0, 12], 24, 16, False), F16, 8)
    probe = normal(rows, 16, F16, g)
    dx = padded(rows, 24, F16)
    dw, db = torch.empty(3, 16, 24, device="cuda"), torch.empty(3, 16, device="cuda")
    gs.expert_linear_backward(probe, x, w, offsets, dx=dx, dw=dw, db=db)

    def loss(x, w, bias):
        out = padded(rows, 16, F16)
        gs.expert_linear(x, w, offsets, out, bias=bias)
        return float((out.double() * probe.double()).sum())
    for t, grad in ((x, dx), (w, dw), (bias, db)):
        direction = torch.randn(t.shape, generator=g, device="cuda")
        up, down = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda"), torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
        up.copy_(t.float() + 0.25 * direction)
        down.copy_(t.float() - 0.25 * direction)
        args = [[z if q is t else q for q in (x, w, bias)] for z in (up, down)]
        moved = loss(*args[0]) - loss(*args[1])
        want = float((grad.double() * (up.double() - down.double())).sum())
        # linear in each argument: only the rounding of the outputs (2^-11 of values of order 4, rows * 16 of
        # them, random) and of the float16 gradient remain
        assert abs(moved - want) <= 4 * 2.0 ** -11 * 4 * math.sqrt(rows * 16) + 2.0 ** -10 * abs(want)


def test_linear_infinities_stay_in_their_rows(gs):
    for case in (([70, 33, 60], 200, 136, False), ([70, 33, 60], 64, 64, True)):
        counts, i, o, gather = case
        g, offsets, rows, row_token, x, w, bias = product_inputs(case, BF16, 12)
        dz = normal(rows, o, BF16, g)
        if not gather:
            x[75], x[80, 3] = math.inf, math.nan             # rows of expert 1
        dz[75, 0], dz[80] = math.nan, math.inf
        w[1, 0] = math.nan
        out, dx = padded(rows, o, BF16), padded(rows, i, BF16)
        dw, db = torch.empty(3, o, i, device="cuda"), torch.empty(3, o, device="cuda")
        gs.expert_linear(x, w, offsets, out, bias=bias, row_token=row_token)
        gs.expert_linear_backward(dz, x, w, offsets, dx=dx, dw=dw, db=db, row_token=row_token)
        for t in (out, dx):
            assert torch.isfinite(t[:70]).all() and torch.isfinite(t[103:]).all()
            assert not torch.isfinite(t[70:103]).all()
        for t in (dw, db):
            assert torch.isfinite(t[0]).all() and torch.isfinite(t[2]).all() and not torch.isfinite(t[1]).all()
        assert torch.isnan(out[70:103, 0]).all() and torch.isfinite(out[70:75, 1:]).all()


def test_linear_bad_indices_never_leave_the_buffers(gs):
    g, offsets, rows, row_token, x, w, bias = product_inputs(([40, 30], 64, 64, True), BF16, 13)
    row_token[3], row_token[50] = -5, x.shape[0] + 1000
    out = padded(rows, 64, BF16)
    gs.expert_linear(x, w, offsets, out, row_token=row_token)
    assert gs.device_status() == BAD_VALUE
    clamped = row_token.clamp(0, x.shape[0] - 1)
    want = padded(rows, 64, BF16)
    gs.expert_linear(x, w, offsets, want, row_token=clamped)
    assert torch.equal(out, want) and gs.device_status() == 0
    dz = normal(rows, 64, BF16, g)
    dws = [torch.empty(2, 64, 64, device="cuda") for _ in range(2)]
    for t, d in zip((row_token, clamped), dws):
        gs.expert_linear_backward(dz, x, w, offsets, dw=d, row_token=t)
    assert torch.equal(*dws) and gs.device_status() == BAD_VALUE
    # offsets past the rows are clamped
    wild = torch.tensor([-7, 40, 10 ** 9], dtype=torch.int32, device="cuda")
    tame = torch.tensor([0, 40, rows], dtype=torch.int32, device="cuda")
    outs = [padded(rows, 64, BF16) for _ in range(2)]
    for t, d in zip((wild, tame), outs):
        gs.expert_linear(x, w, t, d, row_token=clamped)
    assert torch.equal(*outs)


def test_linear_long_segments(gs):
    """Contractions of tens of thousands of rows, one expert holding nearly all."""
    g, offsets, rows, row_token, x, w, bias = product_inputs(([60000, 3, 4001], 96, 64, False), BF16, 15)
    dz = normal(rows, 64, BF16, g)
    dw, db = torch.empty(3, 64, 96, device="cuda"), torch.empty(3, 64, device="cuda")
    gs.expert_linear_backward(dz, x, w, offsets, dw=dw, db=db)
    for e, r in segments(offsets):
        want = dz[r].double().T @ x[r].double()
        # random signs: the error of a sum in float grows with its root, here held to 2^-19 of the whole
        assert float((dw[e].double() - want).norm() / want.norm()) < 2.0 ** -19
        assert float((db[e].double() - dz[r].double().sum(0)).norm() / dz[r].double().sum(0).norm()) < 2.0 ** -19
    again = [torch.empty_like(dw), torch.empty_like(db)]
    gs.expert_linear_backward(dz, x, w, offsets, dw=again[0], db=again[1])
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)


# ---- combination ------------------------------------------------------------------------------

@pytest.mark.parametrize("features", [1, 7, 8, 9, 40, 129, 256, 1000, 1024, 2500])
@pytest.mark.parametrize("k", [1, 2, 7, 16])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_combine(gs, features, k, dtype):
    for n in (1, 75):
        g = gen(features * 31 + k)
        rows = n * k + 3
        token_row = torch.randperm(rows, generator=g, device="cuda")[: n * k].view(n, k).to(torch.int32)
        token_row[torch.rand(n, k, generator=g, device="cuda") < 0.2] = -1
        if n > 1:
            token_row[5] = -1
        y, weight = normal(rows, features, dtype, g, extra=1), torch.randn(n, k, generator=g, device="cuda")
        there = token_row >= 0
        yr = torch.where(there[..., None], y[token_row.clamp_min(0).long()].double(), 0.0)
        for w in (weight, None):
            wd = torch.ones_like(weight).double() if w is None else w.double()
            want, mag = (yr * wd[..., None]).sum(1), (yr * wd[..., None]).abs().sum(1)
            for out_dtype in (dtype, F32):
                out = padded(n, features, out_dtype, extra=1)
                gs.expert_combine(y, token_row, out, weight=w)
                close(out, want, (k + 8) * 2.0 ** -23 * mag + UNIT[out_dtype] * want.abs() + (2.0 ** -25 if out_dtype is F16 else 0))
                assert torch.isnan(rest(out)).all()
                for relu in (False, True):
                    d_out = normal(n, features, out_dtype, g)
                    dy, dw = padded(rows, features, dtype), torch.full((n, k), math.nan, device="cuda")
                    gs.expert_combine_backward(d_out, y, token_row, dy=dy, weight=w, d_weight=dw, relu=relu)
                    dd = d_out.double()[:, None, :]
                    close(dw, (yr * dd).sum(2), (features + 8) * 2.0 ** -23 * (yr * dd).abs().sum(2) + 1e-30)
                    wdy = torch.where(yr > 0, wd[..., None] * dd, 0.0) if relu else wd[..., None] * dd
                    got = dy[token_row.clamp_min(0).long()]
                    close(got[there], wdy[there], (UNIT[dtype] + 2.0 ** -23) * wdy[there].abs() + 2.0 ** -25)
                    untouched = torch.ones(rows, dtype=torch.bool, device="cuda")
                    untouched[token_row[there].long()] = False
                    assert torch.isnan(dy[untouched]).all() and torch.isnan(rest(dy)).all() if features % 8 else True
                    only = torch.empty_like(dw)
                    gs.expert_combine_backward(d_out, y, token_row, d_weight=only, weight=w)
                    assert torch.equal(only, dw)
    assert gs.device_status() == 0


def test_combine_leaves_out_rows_out_of_range(gs):
    y = normal(10, 64, BF16, gen(1))
    token_row = torch.tensor([[0, 10], [-3, 4]], dtype=torch.int32, device="cuda")
    out = padded(2, 64, BF16)
    gs.expert_combine(y, token_row, out)
    assert gs.device_status() == BAD_VALUE
    assert torch.equal(out[0], y[0]) and torch.equal(out[1], y[4])
    dy = padded(10, 64, BF16)
    dw = torch.empty(2, 2, device="cuda")
    gs.expert_combine_backward(out, y, token_row, dy=dy, d_weight=dw)
    assert gs.device_status() == BAD_VALUE and dw[0, 1] == 0 and dw[1, 0] == 0
    assert torch.equal(dy[4], out[1]) and torch.isnan(dy[1]).all()


# ---- clipping ---------------------------------------------------------------------------------

def check_clip(gs, grads, max_norm, outs=None):
    before = [g.clone() for g in grads]
    norm = torch.empty(1, device="cuda")
    gs.clip_grad_norm(grads, max_norm, norm, outs=outs)
    want = math.sqrt(sum(float((b.double() ** 2).sum()) for b in before))
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    f = min(1.0, max_norm / (want + 1e-6))
    for b, o in zip(before, grads if outs is None else outs):
        ref = b.double() * f
        close(o, ref, (UNIT[o.dtype] + 2.0 ** -21) * ref.abs() + (2.0 ** -25 if o.dtype is F16 else 1e-40))
    if outs is not None:
        for b, g in zip(before, grads):
            assert torch.equal(b, g)


@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F16,), (F32, BF16, F16)], ids=str)
@pytest.mark.parametrize("max_norm", [0.0, 0.7, 1e9, math.inf])
def test_clip(gs, dtypes, max_norm):
    g = gen(4)
    sizes = [1, 2, 3, 0, 8, 17, 1000, 4096, 70001, 33, 5]
    flat = {d: torch.zeros(2 * sum(sizes) + 100, dtype=d, device="cuda") for d in dtypes}
    grads, outs, at = [], [], dict.fromkeys(dtypes, 0)
    for j, n in enumerate(sizes):                            # views into one flat buffer, at every alignment
        d = dtypes[j % len(dtypes)]
        t = flat[d][at[d]:at[d] + n]
        t.copy_(torch.randn(n, generator=g, device="cuda") * 0.05)
        grads.append(t)
        outs.append(flat[d][sum(sizes) + 50 + at[d] + j % 2:][:n])
        at[d] += n
    check_clip(gs, grads, max_norm, [torch.empty_like(t) for t in grads])
    other = [torch.zeros(n + 9, dtype=t.dtype, device="cuda")[k % 5:][:n] for k, (n, t) in enumerate(zip(sizes, grads))]
    check_clip(gs, grads, max_norm, other)
    norm = torch.empty(1, device="cuda")
    before = [t.clone() for t in grads]
    gs.clip_grad_norm(grads, max_norm, norm, write=False)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    check_clip(gs, grads, max_norm)                          # in place
    assert gs.device_status() == 0


def test_clip_many_tensors_and_large_ones(gs):
    g = gen(5)
    check_clip(gs, [torch.randn(1 + (j * 37) % 91, generator=g, device="cuda") for j in range(1500)], 1.0)
    check_clip(gs, [torch.randn(9_000_003, generator=g, device="cuda").to(BF16), torch.randn(6_000_001, generator=g, device="cuda")], 3.0)
    norm = torch.full((1,), 5.0, device="cuda")
    gs.clip_grad_norm([], 1.0, norm)
    assert float(norm) == 0.0
    assert gs.device_status() == 0


def test_clip_extreme_values(gs):
    big = [torch.full((100,), 2e37, device="cuda"), torch.full((7,), -1e37, device="cuda")]
    check_clip(gs, big, 1.0)
    tiny = [torch.full((10000,), 1e-30, device="cuda")]
    norm = torch.empty(1, device="cuda")
    gs.clip_grad_norm(tiny, 1.0, norm)
    assert abs(float(norm) - 1e-28) < 1e-34
    assert gs.device_status() == 0
    for v in (math.inf, math.nan, -math.inf):
        t = [torch.randn(5000, device="cuda"), torch.tensor([1.0, v, 2.0], device="cuda")]
        before = [x.clone() for x in t]
        gs.clip_grad_norm(t, 1.0, norm)
        assert not math.isfinite(float(norm)) and gs.device_status() == BAD_VALUE
        assert torch.equal(t[0], before[0]) and torch.equal(torch.isnan(t[1]), torch.isnan(before[1]))


# ---- streams, refusals ------------------------------------------------------------------------

def test_operators_on_another_stream_and_in_a_graph(gs):
    """A whole layer on a side stream, and captured in a graph and replayed: the same results."""
    from paper_2605_16867_b200 import ExpertRouter
    g = gen(21)
    n, e, k, i, o = 300, 9, 2, 128, 72
    logits = torch.randn(n, e, generator=g, device="cuda")
    x, d = normal(n, i, BF16, g), normal(n, o, BF16, g)
    w = (torch.randn(e, o, i, generator=g, device="cuda") * i ** -0.5).to(BF16)
    router = ExpertRouter(e, k)
    i32 = dict(dtype=torch.int32, device="cuda")

    def buffers():
        return dict(expert=torch.zeros(n, k, **i32), weight=torch.zeros(n, k, device="cuda"), offsets=torch.zeros(e + 1, **i32),
                    row_token=torch.zeros(n * k, **i32), token_row=torch.zeros(n, k, **i32), h=padded(n * k, o, BF16, 0.0),
                    y=padded(n, o, BF16, 0.0), dh=padded(n * k, o, BF16, 0.0), dwt=torch.zeros(n, k, device="cuda"),
                    dl=torch.zeros(n, e, device="cuda"), dw=torch.zeros(e, o, i, device="cuda"), db=torch.zeros(e, o, device="cuda"),
                    norm=torch.zeros(1, device="cuda"))

    def layer(b, stream=None):
        gs.expert_route(logits, router, b["expert"], b["weight"], b["offsets"], b["row_token"], b["token_row"], stream=stream)
        gs.expert_linear(x, w, b["offsets"], b["h"], row_token=b["row_token"], relu=True, stream=stream)
        gs.expert_combine(b["h"], b["token_row"], b["y"], weight=b["weight"], stream=stream)
        gs.expert_combine_backward(d, b["h"], b["token_row"], dy=b["dh"], weight=b["weight"], d_weight=b["dwt"], relu=True, stream=stream)
        gs.expert_linear_backward(b["dh"], x, w, b["offsets"], dw=b["dw"], db=b["db"], row_token=b["row_token"], stream=stream)
        gs.expert_route_backward(logits, router, b["expert"], b["dwt"], b["dl"], stream=stream)
        gs.clip_grad_norm([b["dw"], b["db"]], 0.5, b["norm"], stream=stream)
    want = buffers()
    layer(want)
    torch.cuda.synchronize()
    assert 0.4 < math.sqrt(float(want["dw"].double().square().sum() + want["db"].double().square().sum())) < 0.6
    side, got = torch.cuda.Stream(), buffers()
    side.wait_stream(torch.cuda.current_stream())
    layer(got, side)
    side.synchronize()
    assert all(torch.equal(want[k], got[k]) for k in want)
    replayed = buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(replayed)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[k], replayed[k]) for k in want)
    assert gs.device_status() == 0


def test_refusals(gs):
    from paper_2605_16867_b200 import ExpertRouter, GoodServeError
    x = torch.zeros(4, 9, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")

    def outs(k, e=9):
        return [torch.zeros(4, k, **i32), torch.zeros(4, k, device="cuda"), torch.zeros(e + 1, **i32),
                torch.zeros(4 * k, **i32), torch.zeros(4, k, **i32)]

    def refused(code, call):
        before = gs.launch_count()
        with pytest.raises(GoodServeError) as err:
            call()
        assert err.value.code == code
        assert gs.launch_count() == before
    for router in (ExpertRouter(9, 0), ExpertRouter(9, 10), ExpertRouter(9, 2, n_groups=2), ExpertRouter(9, 4, n_groups=3, top_groups=1),
                   ExpertRouter(9, 2, n_groups=3, top_groups=4), ExpertRouter(9, 2, n_groups=3, top_groups=2, group_top=3),
                   ExpertRouter(9, 2, scale=math.nan), ExpertRouter(9, 2, n_groups=0)):
        refused(-1, lambda: gs.expert_route(x, router, *outs(router.top_k)))
    wide = torch.zeros(4, 600, device="cuda")
    refused(-1, lambda: gs.expert_route(wide, ExpertRouter(600, 2), *outs(2, 600)))
    router = ExpertRouter(9, 2)
    refused(-1, lambda: gs.expert_route(x, router, *outs(2)[:3]))                   # an order without its rows
    refused(-4, lambda: gs.expert_route(torch.zeros(5, 9, device="cuda").view(-1)[1:37].view(4, 9), router, *outs(2)))
    with pytest.raises(ValueError):
        ExpertRouter(9, 2, score="tanh")
    with pytest.raises(TypeError):
        gs.expert_route(x.int(), router, *outs(2))
    with pytest.raises(ValueError):
        gs.expert_route(x, ExpertRouter(8, 2), *outs(2, 8))
    with pytest.raises(TypeError):
        gs.expert_route(x.cpu(), router, *outs(2))

    h = torch.zeros(4, 16, dtype=BF16, device="cuda")
    w = torch.zeros(3, 8, 16, dtype=BF16, device="cuda")
    off = torch.zeros(4, **i32)
    out = torch.zeros(4, 8, dtype=BF16, device="cuda")
    odd = torch.zeros(4, 9, dtype=BF16, device="cuda")
    refused(-4, lambda: gs.expert_linear(h, w, off, odd[:, :8]))                   # row stride of 18 bytes
    refused(-4, lambda: gs.expert_linear(torch.zeros(80, dtype=BF16, device="cuda")[1:65].view(4, 16), w, off, out))
    with pytest.raises(TypeError):
        gs.expert_linear(h, w[:, :7], off, out)                                    # experts not evenly spaced
    with pytest.raises(TypeError):
        gs.expert_linear(h.float(), w.float(), off, out.float())
    with pytest.raises(TypeError):
        gs.expert_linear(h, w.half(), off, out)
    refused(-1, lambda: gs.expert_linear(h[:3], w, off, out))                      # fewer rows of x than of out, no row_token
    refused(-1, lambda: gs.expert_linear_backward(out, h, w, off))                 # nothing asked for
    refused(-1, lambda: gs.expert_linear_backward(out, h, w, off, dx=torch.zeros_like(h), db=torch.zeros(3, 8, device="cuda")))
    with pytest.raises(TypeError):
        gs.expert_linear_backward(out, h, w, off, dw=torch.zeros_like(w))
    rows = torch.zeros(4, 17, **i32)
    refused(-1, lambda: gs.expert_combine(h, rows, torch.zeros(4, 16, dtype=BF16, device="cuda")))
    refused(-1, lambda: gs.expert_combine_backward(torch.zeros(4, 16, dtype=BF16, device="cuda"), h, rows[:, :2].contiguous()))
    with pytest.raises(TypeError):
        gs.expert_combine(h, rows[:, :2].contiguous(), torch.zeros(4, 16, dtype=F16, device="cuda"))
    norm = torch.zeros(1, device="cuda")
    for bad in (-1.0, math.nan):
        refused(-1, lambda: gs.clip_grad_norm([x], bad, norm))
    with pytest.raises(TypeError):
        gs.clip_grad_norm([x.int()], 1.0, norm)
    with pytest.raises(ValueError):
        gs.clip_grad_norm([x], 1.0, norm, outs=[])
    assert gs.device_status() == 0
