"""wcc_gated_forward and wcc_gated_backward against their definitions in 64 bits and against differences (needs an MI355X).  What
fp32 sums lose is bounded in block_util; bf16 results are rounded once, and dg and du on their way into the products."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import ACTS, gated_backward, gated_forward, kept, kept_on_gpu, near
from tests.head_util import TYPES, around, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def inputs(rows, ci, co, t, seed, pad=0, shift=0):
    gen = torch.Generator().manual_seed(seed)
    x = rows_of(torch.randn((rows, ci), generator=gen), TYPES[t], pad, shift)
    dy = rows_of(torch.randn((rows, co), generator=gen), TYPES[t], pad, shift)
    wg, wu = ((torch.randn((co, ci), generator=gen) / math.sqrt(ci)).to(TYPES[t]).cuda() for _ in range(2))
    return x, wg, wu, dy


def desc_of(x, y, act, train):
    rows, ci = x.shape
    return wcc.make_gated_desc(rows, ci, y.shape[1], wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32, ACTS[act], train,
                               ldx=x.stride(0) if rows > 1 else ci, ldy=y.stride(0) if rows > 1 else y.shape[1])


def forward(ctx, x, wg, wu, act, pad=0, shift=0, keep=True):
    rows, co = x.shape[0], wg.shape[0]
    y = rows_of(torch.full((rows, co), 9.0), x.dtype, pad, shift)
    codes = torch.full((2, rows, wcc.kept_room(co)), 77, dtype=torch.int8, device="cuda") if keep else None
    steps = torch.full((2, rows, wcc.kept_room(co) // 32), 77, dtype=torch.uint8, device="cuda") if keep else None
    d = desc_of(x, y, act, False)
    ctx.ensure_workspace(d)
    if ctx._ws is not None:
        ctx._ws.fill_(255)  # whatever an earlier call left: here NaN
    ctx.wcc_gated_forward(d, x, wg, wu, y, codes, steps)
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(y)).all())
    return y, codes, steps


def backward(ctx, x, x_kept, wg, wu, act, dy, gu_kept=None, pad=0, shift=0, want=("dx", "dw_gate", "dw_up")):
    dx = rows_of(torch.full((dy.shape[0], wg.shape[1]), 9.0), dy.dtype, pad, shift)
    out = {"dx": dx, "dw_gate": torch.full_like(wg, 9.0), "dw_up": torch.full_like(wg, 9.0)}
    d = desc_of(dx, dy, act, True)
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_gated_backward(d, x, *(x_kept or (None, None)), wg, wu, *(gu_kept or (None, None)), dy,
                           *[out[k] if k in want else None for k in ("dx", "dw_gate", "dw_up")])
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(dx)).all())
    return out


def kept_near(codes, steps, want):
    """Codes of values known to a bound: each within half a step of the value, the steps those of a largest value within the bound."""
    value, err = want
    rows, width = value.shape
    step = torch.exp2(steps.double().cpu() - 127)
    got = codes.double().cpu() * step.repeat_interleave(32, dim=1)
    assert not bool(got[:, width:].any())
    off = (got[:, :width] - value).abs()
    assert bool((off <= step.repeat_interleave(32, dim=1)[:, :width] / 2 + err).all())
    padded = lambda v: torch.nn.functional.pad(v, (0, codes.shape[1] - width))  # noqa: E731
    low, high = kept(padded((value.abs() - err).clamp(min=0)))[1], kept(padded(value.abs() + err))[1]
    assert bool(((steps.cpu() >= low) & (steps.cpu() <= high)).all())


SIZES = [  # rows, C_in, C_out, padding, shift
    (1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (2, 3, 5, 1, 1), (1, 2048, 520, 0, 0), (3, 512, 96, 0, 0), (7, 129, 63, 0, 3), (16, 256, 128, 8, 0),
    (17, 1024, 272, 0, 0), (33, 1000, 137, 3, 1), (64, 320, 640, 0, 0), (65, 64, 257, 0, 0), (100, 72, 96, 8, 8), (130, 512, 384, 0, 0),
    (257, 200, 300, 0, 0), (300, 256, 520, 8, 0), (520, 640, 264, 0, 0), (600, 96, 48, 0, 1), (1000, 40, 24, 0, 0),
    (2, 4104, 88, 0, 0), (20, 5000, 72, 8, 0), (64, 4360, 33, 0, 0),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(ctx, t, act, size):
    rows, ci, co, pad, shift = size
    x, wg, wu, _ = inputs(rows, ci, co, t, sum(size), pad, shift)
    y, codes, steps = forward(ctx, x, wg, wu, act, pad, shift)
    want = gated_forward(x, wg, wu, act)
    near(y, want["y"], t == "bf16")
    kept_near(codes[0], steps[0], want["g"])
    kept_near(codes[1], steps[1], want["u"])
    assert torch.equal(forward(ctx, x, wg, wu, act, pad, shift, keep=False)[0], y)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(ctx, t, act, size):
    rows, ci, co, pad, shift = size
    x, wg, wu, dy = inputs(rows, ci, co, t, sum(size) + 1, pad, shift)
    got, want = backward(ctx, x, None, wg, wu, act, dy, None, pad, shift), gated_backward(x, wg, wu, act, dy, t == "bf16")
    for k in want:
        near(got[k], want[k], t == "bf16", k)
    *x_kept, values = kept_on_gpu(x)  # x in 8 bits, the projections made again
    got, want = backward(ctx, None, x_kept, wg, wu, act, dy, None, pad, shift), gated_backward(values, wg, wu, act, dy, t == "bf16")
    for k in want:
        near(got[k], want[k], t == "bf16", k + " from x in 8 bits")
    _, codes, steps = forward(ctx, x, wg, wu, act, pad, shift)  # all in 8 bits
    gu = [codes[i].double().cpu()[:, :co] * torch.exp2(steps[i].double().cpu() - 127).repeat_interleave(32, dim=1)[:, :co] for i in (0, 1)]
    got = backward(ctx, None, x_kept, wg, wu, act, dy, (codes, steps), pad, shift)
    want = gated_backward(values, wg, wu, act, dy, t == "bf16", gu)
    for k in want:
        near(got[k], want[k], t == "bf16", k + " from all in 8 bits")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("rows", [3, 150])
def test_other_activations(ctx, t, act, rows):
    """relu's slope jumps at 0: g is kept away from there, by a common part of x and of each line of w_gate."""
    ci, co = 96, 80
    x, wg, wu, dy = inputs(rows, ci, co, t, 5)
    x[:, 0], wg[:, 0] = 16.0, torch.where(torch.arange(co) % 2 == 0, 1.0, -1.0).to(wg.dtype).cuda()
    assert float(gated_forward(x, wg, wu, act)["g"][0].abs().min()) > 1
    near(forward(ctx, x, wg, wu, act)[0], gated_forward(x, wg, wu, act)["y"], t == "bf16")
    got, want = backward(ctx, x, None, wg, wu, act, dy), gated_backward(x, wg, wu, act, dy, t == "bf16")
    for k in want:
        near(got[k], want[k], t == "bf16", k)
    _, codes, steps = forward(ctx, x, wg, wu, act)
    gu = [codes[i].double().cpu()[:, :co] * torch.exp2(steps[i].double().cpu() - 127).repeat_interleave(32, dim=1)[:, :co] for i in (0, 1)]
    got, want = backward(ctx, x, None, wg, wu, act, dy, (codes, steps)), gated_backward(x, wg, wu, act, dy, t == "bf16", gu)
    for k in want:
        near(got[k], want[k], t == "bf16", k)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 200])
def test_some_of_the_gradients(ctx, t, rows):
    """What is not asked for is not written, and its inputs may be missing."""
    x, wg, wu, dy = inputs(rows, 104, 72, t, 6)
    whole = backward(ctx, x, None, wg, wu, "silu", dy)
    for some in (("dx",), ("dw_gate",), ("dw_up",), ("dw_gate", "dw_up")):
        got = backward(ctx, x, None, wg, wu, "silu", dy, want=some)
        for k in whole:
            assert torch.equal(got[k], whole[k]) if k in some else bool((got[k] == 9).all()), (some, k)
    _, codes, steps = forward(ctx, x, wg, wu, "silu")
    whole = backward(ctx, x, None, wg, wu, "silu", dy, (codes, steps))
    d = desc_of(x, dy, "silu", True)
    dx, dg, du = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wg)
    ctx.wcc_gated_backward(d, None, None, None, wg, wu, codes, steps, dy, dx)
    ctx.wcc_gated_backward(d, x, None, None, None, None, codes, steps, dy, None, dg, du)
    assert torch.equal(dx, whole["dx"]) and torch.equal(dg, whole["dw_gate"]) and torch.equal(du, whole["dw_up"])


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 20, 150, 400])
def test_what_is_not_finite_stays_in_its_row(ctx, t, rows):
    x, wg, wu, dy = inputs(rows, 136, 200, t, 7)
    y, codes, steps = forward(ctx, x, wg, wu, "silu")
    dx = backward(ctx, x, None, wg, wu, "silu", dy)["dx"]
    bad = rows - 2
    z = x.clone()
    z[bad, 3] = math.nan
    y2, codes2, steps2 = forward(ctx, z, wg, wu, "silu")
    fine = torch.arange(rows) != bad
    assert torch.equal(y2[fine.cuda()], y[fine.cuda()]) and bool(torch.isnan(y2[bad]).all())
    assert torch.equal(codes2[:, fine.cuda()], codes[:, fine.cuda()]) and bool((steps2[:, bad] == 255).all())
    got = backward(ctx, z, None, wg, wu, "silu", dy)
    assert torch.equal(got["dx"][fine.cuda()], dx[fine.cuda()]) and bool(torch.isnan(got["dx"][bad]).all())
    assert bool(torch.isnan(got["dw_gate"]).all()) and bool(torch.isnan(got["dw_up"]).all())
    again = backward(ctx, x, None, wg, wu, "silu", dy, (codes2, steps2))  # (codes of a row that stand for NaN)
    assert bool(torch.isnan(again["dx"][bad]).all()) and bool(torch.isfinite(again["dx"][fine.cuda()]).all())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 104, 72), (40, 1000, 88), (300, 72, 96), (1500, 64, 200), (700, 1032, 600)], ids=str)
def test_infinite_weights_stay_infinities(ctx, t, size):
    """A weight's infinity, or a row's, by a gradient that is not 0 is an infinity of its sign, whatever the gradient is held as."""
    rows, ci, co = size
    x, wg, wu, dy = inputs(rows, ci, co, t, 11)
    _, codes, steps = forward(ctx, x, wg, wu, "silu")
    clean = backward(ctx, x, None, wg, wu, "silu", dy, (codes, steps))
    wu[3, 5] = math.inf
    got = backward(ctx, x, None, wg, wu, "silu", dy, (codes, steps))
    g = codes[0].double()[:, 3] * torch.exp2(steps[0].double()[:, 0] - 127)
    du = dy[:, 3].double() * g * torch.sigmoid(g)
    assert torch.equal(got["dx"][:, 5][du > 0], torch.full_like(dy[:, 0], math.inf)[du > 0])
    assert torch.equal(got["dx"][:, 5][du < 0], torch.full_like(dy[:, 0], -math.inf)[du < 0])
    others = torch.arange(ci).cuda() != 5
    assert torch.equal(got["dx"][:, others], clean["dx"][:, others])
    x[1, 7] = -math.inf
    got = backward(ctx, x, None, wg, wu, "silu", dy, (codes, steps))
    u = codes[1].double()[1, :co] * torch.exp2(steps[1].double()[1] - 127).repeat_interleave(32)[:co]
    g = codes[0].double()[1, :co] * torch.exp2(steps[0].double()[1] - 127).repeat_interleave(32)[:co]
    p = torch.sigmoid(g)
    du, dg = dy[1].double() * g * p, dy[1].double() * u * p * (1 + g * (1 - p))
    for k, v in (("dw_up", du), ("dw_gate", dg)):
        sure = v.abs() > 1e-30
        assert torch.equal(got[k][:, 7].double()[sure], (-math.inf * v.sign())[sure]), k
        others = torch.arange(ci).cuda() != 7
        assert torch.equal(got[k][:, others], clean[k][:, others])


def test_gradients_against_differences(ctx):
    """sum(y r) along random ways, fp32, steps of 2^-7: second-order terms are 2^-14 times a third derivative below 100, rounding
    2^-24 of a sum of about 300 over 2^-6."""
    x, wg, wu, r = inputs(40, 50, 30, "f32", 8)
    got = backward(ctx, x, None, wg, wu, "gelu", r)
    gen = torch.Generator().manual_seed(9)
    at = {"dx": x, "dw_gate": wg, "dw_up": wu}
    for name, v in at.items():
        way = torch.randn(v.shape, generator=gen).cuda() / math.sqrt(v.numel())
        h = 2.0 ** -7
        side = [float((forward(ctx, *(at | {name: (v + s * h * way).contiguous()}).values(), "gelu")[0].double() * r.double()).sum()) for s in (1, -1)]
        along = float((got[name].double() * way.double()).sum())
        assert abs((side[0] - side[1]) / (2 * h) - along) <= 100 * h * h + 300 * 2.0 ** -18, name


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [2, 300])
def test_graph_stream_and_equal_bits(ctx, t, rows):
    """A whole step captured once and replayed over other inputs: equal to the eager calls bit for bit."""
    ci, co = 192, 160
    x, wg, wu, dy = inputs(rows, ci, co, t, 10)
    y, dx, dwg, dwu = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    keep = lambda *lead: (torch.empty((*lead[:-1], wcc.kept_room(lead[-1])), dtype=torch.int8, device="cuda"),  # noqa: E731
                          torch.empty((*lead[:-1], wcc.kept_room(lead[-1]) // 32), dtype=torch.uint8, device="cuda"))
    xk, gk = keep(rows, ci), keep(2, rows, co)
    d, rd = desc_of(x, y, "silu", True), wcc.make_rows_desc(rows, ci, wcc.BF16 if t == "bf16" else wcc.F32)
    own = wcc.Context(0)
    own.ensure_workspace(d)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        own.wcc_rows_keep(rd, x, *xk)
        own.wcc_gated_forward(d, x, wg, wu, y, *gk)
        own.wcc_gated_backward(d, None, *xk, wg, wu, *gk, dy, dx, dwg, dwu)
    for seed in (20, 21, 22):
        x2, _, _, dy2 = inputs(rows, ci, co, t, seed)
        x.copy_(x2), dy.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        y2, codes, steps = forward(ctx, x, wg, wu, "silu")
        got = backward(ctx, None, kept_on_gpu(x)[:2], wg, wu, "silu", dy, (codes, steps))
        for a, b in ((y, y2), (gk[0], codes), (gk[1], steps), (dx, got["dx"]), (dwg, got["dw_gate"]), (dwu, got["dw_up"])):
            assert torch.equal(a, b)
    own.close()


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_no_rows(ctx, t):
    code = wcc.BF16 if t == "bf16" else wcc.F32
    d = wcc.make_gated_desc(0, 24, 40, code, train=True)
    w = torch.ones((40, 24), dtype=TYPES[t], device="cuda")
    ctx.wcc_gated_forward(d, None, None, None, None)
    dwg, dwu = w.clone(), w.clone()
    ctx.wcc_gated_backward(d, None, None, None, None, None, None, None, None, None, dwg, dwu)
    assert not bool(dwg.any()) and not bool(dwu.any())
