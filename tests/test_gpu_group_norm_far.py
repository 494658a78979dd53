"""wcc_group_norm_forward where the mean is far above the spread (needs an MI355X): y and the statistics are as near as elsewhere, on every
route.

Of z = gamma (x - mean) rstd + beta fp32 loses the rounding of x - mean, rstd, gamma rstd and the sum (6 halves of a step of gamma xh and 3
of beta, with room), and of the mean, a fp32 value and its rest, 2^-48 in each of a few places: 2^-45 |mean| rstd |gamma|.  With the mean
rounded to fp32 alone it would be 2^-24 |mean| rstd |gamma|: 0.01 for 10^4 beside a spread of 0.05.  The variance is off by (number of
values) 2^-53 at most, below fp32's rounding."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import ACTS, NARROW, U, act, act_error, kept, near
from tests.head_util import CODE, TYPES, rows_of

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


SIZES = [  # samples, pixels, C, groups, pixels that are there: registers hold them; chunks joined by the second pass; by a launch of their own
    (2, 100, 16, 4, [100, 37]), (3, 40, 21, 7, [40, 0, 9]), (2, 5000, 24, 4, [5000, 4999]), (1, 20000, 20, 1, None), (2, 4097, 363, 3, [4097, 2050]),
    (1, 3000, 1056, 8, None),
]


def forward(ctx, x, samples, groups, name, gamma, beta, counts, keep):
    rows, C = x.shape
    y, stats = torch.zeros_like(x), torch.empty((samples, groups, 2), device="cuda")
    codes = torch.zeros((rows, wcc.kept_room(C)), dtype=torch.int8, device="cuda") if keep else None
    steps = torch.zeros((rows, wcc.kept_room(C) // 32), dtype=torch.uint8, device="cuda") if keep else None
    d = wcc.make_group_norm_desc(samples, rows // samples, C, groups, CODE["bf16" if x.dtype == torch.bfloat16 else "f32"], ACTS[name], EPS,
                                 ldx=x.stride(0), ldy=C)
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_group_norm_forward(d, x, gamma, beta, counts, y, stats, codes, steps)
    torch.cuda.synchronize()
    return y, stats, codes


def want_of(x, samples, groups, name, gamma, beta, counts):
    """(y, its bound), (statistics, their bound), which rows are there"""
    v = x.double().cpu().view(samples, -1, groups, x.shape[1] // groups)
    n = [v.shape[1]] * samples if counts is None else counts.tolist()
    value, tol, stats = torch.zeros_like(v), torch.zeros_like(v), torch.zeros((samples, groups, 2)).double()
    g, b = (p.double().cpu().view(groups, -1) for p in (gamma, beta))
    eps = float(torch.tensor(EPS, dtype=torch.float32))
    for i in range(samples):
        stats[i, :, 1] = 1 / math.sqrt(eps)
        if n[i] == 0:
            continue
        part = v[i, :n[i]]
        mean = part.mean(dim=(0, 2), keepdim=True)
        rstd = 1 / (((part - mean) ** 2).mean(dim=(0, 2), keepdim=True) + eps).sqrt()
        stats[i, :, 0], stats[i, :, 1] = mean.flatten(), rstd.flatten()
        xh = (part - mean) * rstd
        ez = U * (6 * (xh * g).abs() + 3 * b.abs()) + 2.0 ** -45 * (mean * rstd).abs() * g.abs()
        value[i, :n[i]] = act(xh * g + b, name)[0]
        tol[i, :n[i]] = act_error(xh * g + b, ez)[0]
    there = torch.cat([torch.arange(v.shape[1]) < k for k in n])
    return (value.view(x.shape), tol.view(x.shape)), (stats, 2 * U * stats.abs() + 1e-30), there


@pytest.mark.parametrize("level,spread", [(1e4, 0.05), (-1e3, 0.01), (3e6, 4.0), (0.0, 1.0)])
@pytest.mark.parametrize("name", ["none", "silu"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
def test_small_spreads(ctx, size, name, level, spread):
    samples, pixels, C, groups, counts = size
    gen = torch.Generator().manual_seed(sum(size[:4]))
    x = rows_of(level + spread * torch.randn((samples * pixels, C), generator=gen, dtype=torch.float64), torch.float32, 3)
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), (0.3 * torch.randn(C, generator=gen)).cuda()
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    y, stats, _ = forward(ctx, x, samples, groups, name, gamma, beta, counts, False)
    want, want_stats, there = want_of(x, samples, groups, name, gamma, beta, counts)
    near(y[there.cuda()], (want[0][there], want[1][there]), False, "y")
    near(stats, want_stats, False, "stats")
    y2, stats2, codes = forward(ctx, x, samples, groups, name, gamma, beta, counts, True)
    near(y2[there.cuda()], (want[0][there], want[1][there]), False, "y beside codes")
    near(stats2, want_stats, False, "stats beside codes")
    assert torch.equal(codes.cpu()[there][:9], kept(x[:9])[0])


@pytest.mark.parametrize("first", [0.0, 1e5])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
def test_a_first_pixel_far_from_the_others(ctx, size, first):
    """What the sums are taken from is one of the values, and may be the one that is far from all others."""
    samples, pixels, C, groups, counts = size
    gen = torch.Generator().manual_seed(sum(size[:4]) + 1)
    x = rows_of(1e4 + 0.05 * torch.randn((samples * pixels, C), generator=gen, dtype=torch.float64), torch.float32)
    x[::pixels] = first
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), (0.3 * torch.randn(C, generator=gen)).cuda()
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    y, stats, _ = forward(ctx, x, samples, groups, "none", gamma, beta, counts, False)
    want, want_stats, there = want_of(x, samples, groups, "none", gamma, beta, counts)
    near(y[there.cuda()], (want[0][there], want[1][there]), False, "y")
    near(stats, want_stats, False, "stats")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
def test_large_equal_values(ctx, t, size):
    """A group of one value: variance 0 and y = beta whatever the value."""
    samples, pixels, C, groups, counts = size
    x = rows_of(torch.full((samples * pixels, C), 9984.0), TYPES[t])
    gamma, beta = torch.full((C,), 3.0, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    y, stats, _ = forward(ctx, x, samples, groups, "none", gamma, beta, counts, False)
    want, want_stats, there = want_of(x, samples, groups, "none", gamma, beta, counts)
    near(stats, want_stats, False, "stats")
    off = (y[there.cuda()].double() - beta.double()).abs().cpu()
    assert bool((off <= (NARROW if t == "bf16" else U) * 1.001 * beta.double().abs().cpu() + 1e-37).all())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
def test_in_place(ctx, t, size):
    """y in the place of x, whose first pixels are gone when the chunks are joined: equal bits."""
    samples, pixels, C, groups, counts = size
    gen = torch.Generator().manual_seed(sum(size[:4]) + 2)
    x = rows_of(50 + torch.randn((samples * pixels, C), generator=gen), TYPES[t])
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), (0.3 * torch.randn(C, generator=gen)).cuda()
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    y, stats, _ = forward(ctx, x, samples, groups, "silu", gamma, beta, counts, False)
    d = wcc.make_group_norm_desc(samples, pixels, C, groups, CODE[t], ACTS["silu"], EPS)
    again = torch.empty_like(stats)
    there = want_of(x, samples, groups, "silu", gamma, beta, counts)[2].cuda()
    before = x.clone()
    ctx.wcc_group_norm_forward(d, x, gamma, beta, counts, x, again)
    assert torch.equal(x[there], y[there]) and torch.equal(again, stats) and torch.equal(x[~there], before[~there])
