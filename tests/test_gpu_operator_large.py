"""The length predictor's operators on arrays of more than 2^31 elements: their last rows against the same rows
by themselves."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operators import BF16, F32, clean_status, gen, gs  # noqa: E402, F401

ROWS, WIDTH, LAST = 2_200_003, 1024, 300                     # ROWS * WIDTH is 105 million above 2^31
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def wide(g):
    t = torch.zeros(ROWS, WIDTH, dtype=BF16, device="cuda")
    for part in (t[:LAST], t[-LAST:]):
        part.copy_(torch.randn(LAST, WIDTH, generator=g, device="cuda"))
    return t


def test_combine(gs):  # noqa: F811
    g = gen(1)
    y = wide(g)
    token_row = torch.arange(ROWS, **I32).view(-1, 1)
    weight = torch.rand(ROWS, 1, generator=g, device="cuda")
    out = torch.full_like(y, 7.0)
    gs.expert_combine(y, token_row, out, weight=weight)
    want = (y[-LAST:].float() * weight[-LAST:]).to(BF16)
    assert torch.equal(out[-LAST:], want) and (out[LAST:-LAST] == 0).all()
    dy, d_weight = torch.full_like(y, 7.0), torch.empty_like(weight)
    gs.expert_combine_backward(out, y, token_row, dy=dy, weight=weight, d_weight=d_weight)
    assert torch.equal(dy[-LAST:], (want.float() * weight[-LAST:]).to(BF16)) and (dy[LAST:-LAST] == 0).all()
    exact = (y[-LAST:].double() * want.double()).sum(1, keepdim=True)
    assert ((d_weight[-LAST:].double() - exact).abs() <= (WIDTH + 8) * 2.0 ** -23 * exact).all()
    assert gs.device_status() == 0


def test_products(gs):  # noqa: F811
    g = gen(2)
    x, offsets = wide(g), torch.tensor([0, 5, ROWS], **I32)
    tail = torch.tensor([0, 0, LAST], **I32)
    narrow = torch.randn(2, 24, WIDTH, generator=g, device="cuda").to(BF16)          # WIDTH to 24 and back
    out, alone = (torch.full((n, 24), 7.0, dtype=BF16, device="cuda") for n in (ROWS, LAST))
    gs.expert_linear(x, narrow, offsets, out)
    gs.expert_linear(x[-LAST:], narrow, tail, alone)
    assert torch.equal(out[-LAST:], alone) and (out[LAST:-LAST] == 0).all()
    reverse = torch.arange(ROWS - 1, -1, -1, **I32)                                  # the last tokens first
    gs.expert_linear(x, narrow, offsets, out, row_token=reverse)
    gs.expert_linear(x[-LAST:].flip(0).contiguous(), narrow, torch.tensor([0, 5, LAST], **I32), alone)
    assert torch.equal(out[:LAST], alone)
    dz, dx = torch.full((ROWS, 24), 0.5, dtype=BF16, device="cuda"), torch.full_like(x, 7.0)
    gs.expert_linear_backward(dz, x, narrow, offsets, dx=dx, relu_input=True)
    back = torch.empty(LAST, WIDTH, dtype=BF16, device="cuda")
    gs.expert_linear_backward(dz[-LAST:], x[-LAST:], narrow, tail, dx=back, relu_input=True)
    assert torch.equal(dx[-LAST:], back) and (dx[LAST:-LAST] == 0).all()
    del dx
    dw, db = torch.empty(2, 24, WIDTH, device="cuda"), torch.empty(2, 24, device="cuda")
    for row_token in (None, reverse):
        gs.expert_linear_backward(dz, x, narrow, offsets, dw=dw, db=db, row_token=row_token)
        for e, r in ((0, slice(0, 5)), (1, slice(5, ROWS))):
            rows = x[-5:] if row_token is not None and e == 0 else x[:5] if e == 0 else None
            if rows is None:
                ends = (x[:LAST], x[-LAST:])
                rows = torch.cat([ends[0], ends[1][:-5]] if row_token is not None else [ends[0][5:], ends[1]])
            want = 0.5 * rows.double().sum(0)
            room = (2 * LAST + 768) * 2.0 ** -23 * rows.double().abs().sum(0)
            assert ((dw[e].double() - want).abs() <= room).all()
            assert ((db[e] - 0.5 * (r.stop - r.start)).abs() <= 2.0 ** -22 * (r.stop - r.start)).all()
    del x
    x16 = torch.randn(ROWS, 16, generator=g, device="cuda").to(BF16)
    out = torch.full((ROWS, WIDTH), 7.0, dtype=BF16, device="cuda")
    back = narrow.transpose(1, 2).contiguous()[..., :16].contiguous()
    gs.expert_linear(x16, back, offsets, out)
    alone = torch.empty(LAST, WIDTH, dtype=BF16, device="cuda")
    gs.expert_linear(x16[-LAST:], back, tail, alone)
    assert torch.equal(out[-LAST:], alone)
    assert gs.device_status() == 0


def test_routing(gs):  # noqa: F811
    from paper_2605_16867_b200 import ExpertRouter
    g, e, k = gen(3), 256, 4
    n = ROWS * WIDTH // e
    x = torch.zeros(n, e, dtype=BF16, device="cuda")
    x[-LAST:] = torch.randn(LAST, e, generator=g, device="cuda").to(BF16)
    router = ExpertRouter(e, k)
    expert, weight, offsets = torch.empty(n, k, **I32), torch.empty(n, k, device="cuda"), torch.empty(e + 1, **I32)
    row_token, token_row = torch.empty(n * k, **I32), torch.empty(n, k, **I32)
    gs.expert_route(x, router, expert, weight, offsets, row_token, token_row)
    alone = torch.empty(LAST, k, **I32), torch.empty(LAST, k, device="cuda")
    gs.expert_route(x[-LAST:], router, *alone)
    assert torch.equal(expert[-LAST:], alone[0]) and torch.equal(weight[-LAST:], alone[1])
    assert (expert[:-LAST] == torch.arange(k, **I32)).all()
    counts = torch.bincount(expert.view(-1).long(), minlength=e)
    assert torch.equal(offsets.long(), torch.cat([counts.new_zeros(1), counts.cumsum(0)]))
    rows = token_row.view(-1).long()
    slots = torch.empty_like(rows)
    slots[rows] = torch.arange(n * k, device="cuda")
    assert torch.equal(row_token.long(), slots // k)
    first = expert.view(-1)[slots]
    assert (first[1:] >= first[:-1]).all() and ((slots[1:] > slots[:-1]) | (first[1:] > first[:-1])).all()
    d, d_weight = torch.full_like(x, 7.0), torch.randn(n, k, generator=g, device="cuda")
    gs.expert_route_backward(x, router, expert, d_weight, d)
    back = torch.empty(LAST, e, dtype=BF16, device="cuda")
    gs.expert_route_backward(x[-LAST:], router, alone[0], d_weight[-LAST:].contiguous(), back)
    assert torch.equal(d[-LAST:], back)
    assert gs.device_status() == 0


def test_clipping(gs):  # noqa: F811
    g = wide(gen(4)).view(-1)
    norm = torch.empty(1, device="cuda")
    last = g[-LAST * WIDTH:].clone()
    want = math.sqrt(float(last.double().square().sum()) + float(g[:LAST * WIDTH].double().square().sum()))
    gs.clip_grad_norm([g], 1.0, norm)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    f = torch.tensor(1.0, device="cuda") / (norm + 1e-6)
    assert torch.equal(g[-LAST * WIDTH:], (last.float() * f).to(BF16))
    assert gs.device_status() == 0
