"""wcc_group_norm_forward and wcc_group_norm_backward against their definitions in 64 bits and against differences (needs an
MI355X).  What fp32 loses is bounded value by value in block_util; bf16 results are rounded once more."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import ACTS, group_norm, kept, near
from tests.head_util import CODE, TYPES, around, rows_of

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def inputs(samples, pixels, C, t, seed, pad=0, shift=0, counts=None, spread=0.5):
    gen = torch.Generator().manual_seed(seed)
    rows = samples * pixels
    v = torch.randn((rows, C), generator=gen) * (0.5 + torch.rand(C, generator=gen)) + spread * torch.randn(C, generator=gen)
    x = rows_of(v, TYPES[t], pad, shift)
    dy = rows_of(torch.randn((rows, C), generator=gen), TYPES[t], pad, shift)
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), (0.3 * torch.randn(C, generator=gen)).cuda()
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    return x, gamma, beta, counts, dy


def desc_of(x, y, samples, groups, act):
    rows, C = x.shape
    return wcc.make_group_norm_desc(samples, rows // samples, C, groups, wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32, ACTS[act], EPS,
                                    ldx=x.stride(0) if rows > 1 else C, ldy=y.stride(0) if rows > 1 else C)


def forward(ctx, x, samples, groups, act, gamma, beta, counts, pad=0, shift=0, keep=True):
    rows, C = x.shape
    y = rows_of(torch.full((rows, C), 9.0), x.dtype, pad, shift)
    out = {"y": y, "stats": torch.full((samples, groups, 2), 9.0, device="cuda"),
           "codes": torch.full((rows, wcc.kept_room(C)), 77, dtype=torch.int8, device="cuda") if keep else None,
           "steps": torch.full((rows, wcc.kept_room(C) // 32), 77, dtype=torch.uint8, device="cuda") if keep else None}
    d = desc_of(x, y, samples, groups, act)
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)  # whatever an earlier call left: here NaN
    ctx.wcc_group_norm_forward(d, x, gamma, beta, counts, y, out["stats"], out["codes"], out["steps"])
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(y)).all())
    return out


def backward(ctx, x, kept_x, samples, groups, act, gamma, beta, counts, stats, dy, pad=0, shift=0, want=("dx", "dgamma", "dbeta")):
    rows, C = dy.shape
    dx = rows_of(torch.full((rows, C), 9.0), dy.dtype, pad, shift)
    out = {"dx": dx, "dgamma": torch.full((C,), 9.0, device="cuda"), "dbeta": torch.full((C,), 9.0, device="cuda")}
    d = desc_of(dx, dy, samples, groups, act)
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_group_norm_backward(d, x, *(kept_x or (None, None)), gamma, beta, counts, stats, dy,
                                *[out[k] if k in want else None for k in ("dx", "dgamma", "dbeta")])
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(dx)).all())
    return out


def there(counts, samples, pixels):
    n = [pixels] * samples if counts is None else [min(max(int(c), 0), pixels) for c in counts]
    return torch.cat([torch.arange(pixels) < k for k in n])


def rows_near(got, want, mask, narrow, what):
    near(got[mask.to(got.device)], (want[0][mask], want[1][mask]), narrow, what)
    assert bool((got[~mask.to(got.device)] == 9).all()), what  # rows that are not there stay as they were


SIZES = [  # samples, pixels, C, groups, padding, shift, counts
    (1, 1, 1, 1, 0, 0, None), (1, 64, 1, 1, 0, 0, None), (2, 50, 3, 1, 1, 1, None), (1, 256, 96, 8, 0, 0, None), (3, 100, 40, 5, 0, 0, None),
    (2, 37, 24, 24, 3, 2, None), (4, 33, 96, 32, 0, 0, [33, 5, 0, 40]), (2, 500, 64, 2, 8, 0, [500, 123]), (1, 3000, 32, 4, 0, 0, None),
    (2, 20, 2200, 11, 0, 0, None), (1, 40, 700, 1, 5, 1, None), (5, 1, 512, 2, 0, 0, [1, 0, 1, -3, 1]), (1, 5000, 20, 4, 0, 8, None),
    (40, 70, 16, 2, 0, 0, None), (2, 4097, 360, 3, 0, 0, [4097, 2050]), (1, 900, 1200, 1, 8, 0, None),  # (many pairs of sums to a group)
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_both_directions(ctx, t, act, size):
    samples, pixels, C, groups, pad, shift, counts = size
    x, gamma, beta, counts, dy = inputs(samples, pixels, C, t, sum(size[:4]), pad, shift, counts)
    got = forward(ctx, x, samples, groups, act, gamma, beta, counts, pad, shift)
    mask = there(counts, samples, pixels)
    codes, steps, values = kept(x)
    want = group_norm(x, samples, groups, gamma, beta, counts, EPS, act, dy)
    rows_near(got["y"], want["y"], mask, t == "bf16", "y")
    near(got["stats"], want["stats"], False, "stats")
    assert torch.equal(got["codes"].cpu()[mask], codes[mask]) and torch.equal(got["steps"].cpu()[mask], steps[mask])
    assert bool((got["codes"].cpu()[~mask] == 77).all()) and bool((got["steps"].cpu()[~mask] == 77).all())
    grads = backward(ctx, x, None, samples, groups, act, gamma, beta, counts, got["stats"], dy, pad, shift)
    rows_near(grads["dx"], want["dx"], mask, t == "bf16", "dx")
    for k in ("dgamma", "dbeta"):
        near(grads[k], want[k], False, k)
    want = group_norm(x, samples, groups, gamma, beta, counts, EPS, act, dy, values)
    grads = backward(ctx, None, (got["codes"], got["steps"]), samples, groups, act, gamma, beta, counts, got["stats"], dy, pad, shift)
    rows_near(grads["dx"], want["dx"], mask, t == "bf16", "dx from codes")
    for k in ("dgamma", "dbeta"):
        near(grads[k], want[k], False, k + " from codes")


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_relu(ctx, t):
    """z is kept away from 0, where the slope jumps: gamma is small and beta is not."""
    x, gamma, beta, _, dy = inputs(2, 60, 48, t, 5)
    gamma = gamma * 0.02
    beta = torch.where(beta > 0, 1.0, -1.0)
    got = forward(ctx, x, 2, 6, "relu", gamma, beta, None)
    want = group_norm(x, 2, 6, gamma, beta, None, EPS, "relu", dy)
    near(got["y"], want["y"], t == "bf16")
    grads = backward(ctx, x, None, 2, 6, "relu", gamma, beta, None, got["stats"], dy)
    for k in ("dx", "dgamma", "dbeta"):
        near(grads[k], want[k], t == "bf16" and k == "dx", k)
    zero = torch.zeros_like(beta)  # z = 0 throughout: value and slope 0
    got = forward(ctx, x, 2, 6, "relu", zero, zero, None)
    grads = backward(ctx, x, None, 2, 6, "relu", zero, zero, None, got["stats"], dy)
    assert not bool(got["y"].any()) and not any(bool(grads[k].any()) for k in grads)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_optional_parts(ctx, t):
    """Without gamma, beta, stats and codes; some of the gradients only; results in place of inputs."""
    x, gamma, beta, _, dy = inputs(2, 45, 72, t, 6)
    want = group_norm(x, 2, 9, None, None, None, EPS, "silu", dy)
    y = torch.empty_like(x)
    d = desc_of(x, y, 2, 9, "silu")
    ctx.ensure_workspace(d)
    ctx.wcc_group_norm_forward(d, x, None, None, None, y)
    near(y, want["y"], t == "bf16")
    stats = forward(ctx, x, 2, 9, "silu", None, None, None)["stats"]
    for some in (("dx",), ("dgamma",), ("dbeta",), ("dgamma", "dbeta")):
        got = backward(ctx, x, None, 2, 9, "silu", None, None, None, stats, dy, want=some)
        for k in ("dx", "dgamma", "dbeta"):
            if k in some:
                near(got[k], want[k], t == "bf16" and k == "dx", k)
            else:
                assert bool((got[k] == 9).all())
    dxs = backward(ctx, x, None, 2, 9, "silu", gamma, beta, None, stats, dy)["dx"]
    plain = forward(ctx, x, 2, 9, "silu", gamma, beta, None)
    z = x.clone()
    ctx.wcc_group_norm_forward(d, z, gamma, beta, None, z)
    assert torch.equal(z, plain["y"])
    g = dy.clone()
    ctx.wcc_group_norm_backward(d, x, None, None, gamma, beta, None, stats, g, g)
    assert torch.equal(g, dxs)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_means_far_above_the_spread(ctx, t):
    """Means of 300 (bf16: the values' own rounding is then their spread) and of 10^4 beside a spread of about 1."""
    for level in (300.0, 1e4):
        x, gamma, beta, _, dy = inputs(2, 400, 16, t, 7, spread=level)
        got = forward(ctx, x, 2, 4, "none", gamma, beta, None)
        want = group_norm(x, 2, 4, gamma, beta, None, EPS, "none", dy)
        near(got["y"], want["y"], t == "bf16")
        near(got["stats"], want["stats"], False)
        got = backward(ctx, x, None, 2, 4, "none", gamma, beta, None, got["stats"], dy)
        near(got["dx"], want["dx"], t == "bf16")


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_equal_values(ctx, t):
    """A group without spread: y = act(beta) and rstd = 1 / sqrt(eps)."""
    x = rows_of(torch.full((90, 32), 0.75), TYPES[t])
    gamma, beta = torch.ones(32, device="cuda"), torch.linspace(-1, 1, 32, device="cuda")
    got = forward(ctx, x, 3, 4, "none", gamma, beta, None)
    want = group_norm(x, 3, 4, gamma, beta, None, EPS, "none")
    near(got["y"], want["y"], t == "bf16")
    near(got["stats"], want["stats"], False)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_group(ctx, t):
    x, gamma, beta, _, dy = inputs(3, 50, 64, t, 8)
    clean = forward(ctx, x, 3, 4, "silu", gamma, beta, None)
    first = backward(ctx, x, None, 3, 4, "silu", gamma, beta, None, clean["stats"], dy)
    z = x.clone()
    z[60, 20], z[3, 50] = math.nan, math.inf  # sample 1, group 1; sample 0, group 3
    got = forward(ctx, z, 3, 4, "silu", gamma, beta, None)
    bad = torch.zeros((3, 50, 64), dtype=torch.bool)
    bad[1, :, 16:32], bad[0, :, 48:] = True, True
    bad = bad.view(150, 64).cuda()
    assert bool(torch.isnan(got["y"][bad]).all()) and torch.equal(got["y"][~bad], clean["y"][~bad])
    grads = backward(ctx, z, None, 3, 4, "silu", gamma, beta, None, got["stats"], dy)
    assert bool(torch.isnan(grads["dx"][bad]).all()) and torch.equal(grads["dx"][~bad], first["dx"][~bad])
    fine = torch.ones(64, dtype=torch.bool)
    fine[16:32], fine[48:] = False, False
    for k in ("dgamma", "dbeta"):
        assert torch.equal(grads[k].cpu()[fine], first[k].cpu()[fine]) and bool(torch.isnan(grads[k].cpu()[~fine]).all())


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_rows_that_are_not_there_are_not_read(ctx, t):
    x, gamma, beta, counts, dy = inputs(4, 30, 48, t, 9, counts=[30, 7, 0, 21])
    clean = forward(ctx, x, 4, 3, "gelu", gamma, beta, counts)
    first = backward(ctx, x, None, 4, 3, "gelu", gamma, beta, counts, clean["stats"], dy)
    gone = ~there(counts, 4, 30).cuda()
    x[gone], dy[gone] = math.nan, math.nan
    got = forward(ctx, x, 4, 3, "gelu", gamma, beta, counts)
    again = backward(ctx, x, None, 4, 3, "gelu", gamma, beta, counts, got["stats"], dy)
    for k in ("y", "stats", "codes", "steps"):
        assert torch.equal(got[k], clean[k]), k
    for k in ("dx", "dgamma", "dbeta"):
        assert torch.equal(again[k], first[k]), k


def test_gradients_against_differences(ctx):
    """The kernel's gradients of sum(y r) against central differences of the kernel's own y, in fp32 with steps of 2^-8: what the
    second-order term leaves, 2^-16 times a third derivative of a few hundred, and rounding, 2^-24 of a sum of 200 over 2^-7."""
    samples, pixels, C, groups = 2, 25, 12, 3
    x, gamma, beta, counts, r = inputs(samples, pixels, C, "f32", 10, counts=[25, 14])
    mask = there(counts, samples, pixels).cuda()

    def loss(x, gamma, beta):
        y = forward(ctx, x, samples, groups, "silu", gamma, beta, counts)["y"]
        return float((y.double() * r.double())[mask].sum())
    stats = forward(ctx, x, samples, groups, "silu", gamma, beta, counts)["stats"]
    got = backward(ctx, x, None, samples, groups, "silu", gamma, beta, counts, stats, r)
    gen = torch.Generator().manual_seed(11)
    for name, v in (("dx", x), ("dgamma", gamma), ("dbeta", beta)):
        way = torch.randn(v.shape, generator=gen).cuda() / math.sqrt(v.numel())
        h = 2.0 ** -8
        moved = [{"dx": x, "dgamma": gamma, "dbeta": beta} | {name: v + s * h * way} for s in (1, -1)]
        diff = (loss(*[moved[0][k] for k in ("dx", "dgamma", "dbeta")]) - loss(*[moved[1][k] for k in ("dx", "dgamma", "dbeta")])) / (2 * h)
        along = (got[name].double() * way.double())
        along = float(along[mask].sum() if name == "dx" else along.sum())
        assert abs(diff - along) <= 300 * h * h + 200 * 2.0 ** -17, (name, diff, along)


def test_graph_stream_and_equal_bits(ctx):
    """Captured once with its backward pass, replayed over other inputs, on a stream of its own: equal to the eager calls bit for bit."""
    samples, pixels, C, groups = 3, 700, 64, 8
    x, gamma, beta, _, dy = inputs(samples, pixels, C, "bf16", 12)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    stats = torch.empty((samples, groups, 2), device="cuda")
    codes, steps = torch.empty((x.shape[0], 64), dtype=torch.int8, device="cuda"), torch.empty((x.shape[0], 2), dtype=torch.uint8, device="cuda")
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    d = desc_of(x, y, samples, groups, "silu")
    own = wcc.Context(0)
    own.ensure_workspace(d)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        own.wcc_group_norm_forward(d, x, gamma, beta, None, y, stats, codes, steps)
        own.wcc_group_norm_backward(d, None, codes, steps, gamma, beta, None, stats, dy, dx, dgamma, dbeta)
    for seed in (20, 21, 22):
        x2, _, _, _, dy2 = inputs(samples, pixels, C, "bf16", seed)
        x.copy_(x2), dy.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        got = forward(ctx, x, samples, groups, "silu", gamma, beta, None)
        grads = backward(ctx, None, (got["codes"], got["steps"]), samples, groups, "silu", gamma, beta, None, got["stats"], dy)
        for a, b in ((y, got["y"]), (stats, got["stats"]), (codes, got["codes"]), (dx, grads["dx"]), (dgamma, grads["dgamma"]), (dbeta, grads["dbeta"])):
            assert torch.equal(a, b)
    own.close()


def test_pixels_behind_32_bits(ctx):
    """A sample of more than 2^31 values: its last pixels, and statistics over all of them."""
    pixels, C = (1 << 25) + 3, 65
    x = torch.full((pixels, C), 1.0, dtype=torch.bfloat16, device="cuda")
    x[::2] = -1.0  # (one pixel more at -1 than at 1)
    y = torch.zeros_like(x)
    d = wcc.make_group_norm_desc(1, pixels, C, 1, wcc.BF16, wcc.ACT_NONE, EPS)
    ctx.ensure_workspace(d)
    stats = torch.empty((1, 1, 2), device="cuda")
    ctx.wcc_group_norm_forward(d, x, None, None, None, y, stats)
    assert bool((y == x).all())  # (mean -3e-8, variance 1: bf16 has nothing of the difference)
    assert abs(float(stats[0, 0, 0]) + 1 / pixels) < 1e-12
    dx, dgamma, dbeta = torch.zeros_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    y[-1] = 3.0
    ctx.wcc_group_norm_backward(d, x, None, None, None, None, None, stats, y, dx, dgamma, dbeta)
    assert float(dx[-1, 0]) == pytest.approx(4.0, rel=2.0 ** -8) and float(dbeta[7]) == pytest.approx(3.0, abs=1e-3)
    assert float(dgamma[64]) == pytest.approx((pixels - 4) / math.sqrt(1 + EPS), rel=1e-6)  # (xh is x rstd)


def test_no_samples(ctx):
    d = wcc.make_group_norm_desc(0, 5, 8, 2, wcc.F32)
    ctx.wcc_group_norm_forward(d, None, None, None, None, None)
    ctx.ensure_workspace(d)
    dgamma, dbeta = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    ctx.wcc_group_norm_backward(d, None, None, None, None, None, None, None, None, None, dgamma, dbeta)
    assert not bool(dgamma.any()) and not bool(dbeta.any()) and CODE["f32"] == wcc.F32


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(65, 3, 40, 4), (1500, 2, 24, 3), (300, 1, 520, 1), (70, 1200, 8, 1), (100, 40, 1300, 2)], ids=str)
def test_many_samples(ctx, t, size):
    """More samples than one thread adds up: on maps that registers hold, and on others."""
    samples, pixels, C, groups = size
    x, gamma, beta, _, dy = inputs(samples, pixels, C, t, sum(size))
    got = forward(ctx, x, samples, groups, "silu", gamma, beta, None)
    want = group_norm(x, samples, groups, gamma, beta, None, EPS, "silu", dy)
    near(got["y"], want["y"], t == "bf16")
    for some in (("dx", "dgamma", "dbeta"), ("dgamma", "dbeta")):
        grads = backward(ctx, x, None, samples, groups, "silu", gamma, beta, None, got["stats"], dy, want=some)
        for k in some:
            near(grads[k], want[k], t == "bf16" and k == "dx", k)


HELD = [  # samples, pixels, C, groups: what a workgroup's registers hold, and what is just too large for them
    (2, 4096, 8, 1), (2, 4097, 8, 1), (1, 1024, 32, 4), (1, 1025, 32, 4), (3, 128, 256, 32), (1, 64, 512, 1), (1, 64, 520, 1), (300, 4, 128, 32),
    (2, 2000, 64, 64), (7, 9, 480, 5), (1, 2048, 24, 2), (1, 8192, 4, 4),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", HELD, ids=lambda s: "x".join(map(str, s)))
def test_what_registers_hold(ctx, t, size):
    samples, pixels, C, groups = size
    counts = [pixels, 0, pixels // 2] if samples == 3 else None
    x, gamma, beta, counts, dy = inputs(samples, pixels, C, t, sum(size), 0, 0, counts)
    got = forward(ctx, x, samples, groups, "silu", gamma, beta, counts)
    mask = there(counts, samples, pixels)
    want = group_norm(x, samples, groups, gamma, beta, counts, EPS, "silu", dy)
    rows_near(got["y"], want["y"], mask, t == "bf16", "y")
    near(got["stats"], want["stats"], False, "stats")
    grads = backward(ctx, x, None, samples, groups, "silu", gamma, beta, counts, got["stats"], dy)
    rows_near(grads["dx"], want["dx"], mask, t == "bf16", "dx")
    for k in ("dgamma", "dbeta"):
        near(grads[k], want[k], False, k)
