"""wcc_rows_keep and wcc_rows_restore (needs an MI355X): codes, steps and values are those of the definition, bit for bit."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import kept
from tests.head_util import CODE, TYPES, around, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def keep(ctx, x):
    rows, width = x.shape
    d = wcc.make_rows_desc(rows, width, wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32, ld=x.stride(0) if rows > 1 else width)
    codes = torch.full((rows, wcc.kept_room(width)), 77, dtype=torch.int8, device="cuda")
    steps = torch.full((rows, wcc.kept_room(width) // 32), 77, dtype=torch.uint8, device="cuda")
    ctx.wcc_rows_keep(d, x, codes, steps)
    return codes, steps


def restore(ctx, codes, steps, width, dtype, pad=0, shift=0):
    x = rows_of(torch.full((codes.shape[0], width), 9.0), dtype, pad, shift)
    d = wcc.make_rows_desc(codes.shape[0], width, wcc.BF16 if dtype == torch.bfloat16 else wcc.F32,
                           ld=x.stride(0) if codes.shape[0] > 1 else width)
    ctx.wcc_rows_restore(d, codes, steps, x)
    assert bool(torch.isnan(around(x)).all())
    return x


def check(ctx, values, t, pad=0, shift=0):
    x = rows_of(values, TYPES[t], pad, shift)
    codes, steps = keep(ctx, x)
    want_codes, want_steps, want = kept(x)
    assert torch.equal(steps.cpu(), want_steps)
    assert torch.equal(codes.cpu(), want_codes)
    back = restore(ctx, codes, steps, values.shape[1], TYPES[t], pad, shift)
    assert torch.equal(back.double().cpu().nan_to_num(-5.5e30), want.nan_to_num(-5.5e30))
    other = "f32" if t == "bf16" else "bf16"  # (the values are exact in either type)
    back = restore(ctx, codes, steps, values.shape[1], TYPES[other], pad, shift)
    assert torch.equal(back.double().cpu().nan_to_num(-5.5e30), want.nan_to_num(-5.5e30))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 0, 0), (1, 31, 0, 1), (3, 32, 0, 0), (5, 33, 1, 3), (7, 64, 8, 0), (2, 255, 3, 1), (40, 96, 0, 0),
                                  (9, 1000, 0, 5), (300, 7, 0, 0), (33, 264, 5, 2)], ids=lambda s: "x".join(map(str, s)))
def test_sizes(ctx, t, size):
    rows, width, pad, shift = size
    gen = torch.Generator().manual_seed(sum(size))
    x = torch.randn((rows, width), generator=gen) * torch.exp(3 * torch.randn((rows, 1), generator=gen))
    x[torch.rand((rows, width), generator=gen) < 0.02] *= 50
    check(ctx, x, t, pad, shift)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_borders(ctx, t):
    """Ties, largest values that round to 128 steps, powers of two, signs, zeros."""
    rows = []
    for top in (64.0, 65.0, 127.0, 127.25, 127.5, 127.75, 128.0, 1.0, 1.9921875, 1.984375):
        for scale in (1.0, 2.0 ** -20, 2.0 ** 40, -1.0):
            row = torch.arange(32) * 0.5 - 4.0
            row[0] = top
            rows.append(row * scale)
    rows.append(torch.zeros(32))
    rows.append(-torch.zeros(32))
    check(ctx, torch.stack(rows), t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_ends_of_the_range(ctx, t):
    most = torch.finfo(TYPES[t]).max
    least = torch.finfo(TYPES[t]).tiny
    base = torch.linspace(-1, 1, 32)
    rows = [base * most, base * most * 0.99, base * most / 2, torch.full((32,), -most), base * least, base * least * 64, base * least * 127,
            base * least * 128, base * least * 300, base * least / 4, torch.tensor([least / 8] + [0.0] * 31)]
    check(ctx, torch.stack(rows), t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_blocks_that_are_not_finite(ctx, t):
    """Only the block that holds an infinity or NaN stands for NaN."""
    x = torch.randn((4, 100), generator=torch.Generator().manual_seed(3))
    x[0, 5], x[1, 40], x[2, 99], x[3, 64] = math.inf, -math.inf, math.nan, math.inf
    check(ctx, x, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_kept_again(ctx, t):
    """What has been kept is kept exactly."""
    x = rows_of(torch.randn((50, 200), generator=torch.Generator().manual_seed(4)) * 30, TYPES[t])
    codes, steps = keep(ctx, x)
    back = restore(ctx, codes, steps, 200, TYPES[t])
    again = keep(ctx, back)
    assert torch.equal(again[0], codes) and torch.equal(again[1], steps)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_many_rows_are_kept_row_by_row(ctx, t):
    """More vectors than the launch has threads: each row as by itself."""
    x = rows_of(torch.randn((70001, 129), generator=torch.Generator().manual_seed(5)), TYPES[t], 3)
    codes, steps = keep(ctx, x)
    back = restore(ctx, codes, steps, 129, TYPES[t])
    for r in (0, 1, 30011, 52429, 70000):
        want_codes, want_steps, want = kept(x[r:r + 1])
        assert torch.equal(codes[r:r + 1].cpu(), want_codes) and torch.equal(steps[r:r + 1].cpu(), want_steps)
    step = torch.exp2(steps.double() - 127).repeat_interleave(32, dim=1)[:, :129]
    assert bool(((back.double() - x.double()).abs() <= step / 2).all())


def test_rows_behind_32_bits(ctx):
    """A matrix of more than 2^31 elements, its last rows."""
    rows, width = 1 << 21, 1056
    x = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
    x[:8].normal_(), x[-8:].normal_()
    x[8:-8] = 1.0
    codes, steps = keep(ctx, x)
    back = torch.zeros_like(x)
    d = wcc.make_rows_desc(rows, width, wcc.BF16)
    ctx.wcc_rows_restore(d, codes, steps, back)
    for part in (slice(0, 8), slice(rows - 8, rows)):
        want_codes, want_steps, want = kept(x[part])
        assert torch.equal(codes[part].cpu(), want_codes) and torch.equal(steps[part].cpu(), want_steps)
        assert torch.equal(back[part].double().cpu(), want)
    assert bool((back[8:-8] == 1).all())


def test_graph_and_stream(ctx):
    x = torch.randn((200, 160), device="cuda")
    d = wcc.make_rows_desc(200, 160, wcc.F32)
    codes = torch.empty((200, 160), dtype=torch.int8, device="cuda")
    steps = torch.empty((200, 5), dtype=torch.uint8, device="cuda")
    back = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.wcc_rows_keep(d, x, codes, steps)
        ctx.wcc_rows_restore(d, codes, steps, back)
    for seed in range(3):
        x.copy_(torch.randn((200, 160), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(back.double().cpu(), kept(x)[2])


def test_no_rows(ctx):
    d = wcc.make_rows_desc(0, 40, wcc.BF16)
    ctx.wcc_rows_keep(d, None, None, None)
    ctx.wcc_rows_restore(d, None, None, None)
    assert CODE["bf16"] == wcc.BF16


def test_another_device_is_refused(ctx, monkeypatch):
    """Tensors, or a context, of another device than the current one."""
    x = torch.ones((3, 40), device="cuda")
    d = wcc.make_rows_desc(3, 40, wcc.F32)
    codes, steps = torch.zeros((3, 64), dtype=torch.int8, device="cuda"), torch.zeros((3, 2), dtype=torch.uint8, device="cuda")
    with monkeypatch.context() as m:
        m.setattr(wcc, "_current_device", lambda: 1)
        with pytest.raises(AssertionError, match="the current device"):
            ctx.wcc_rows_keep(d, x, codes, steps)
    with monkeypatch.context() as m:
        m.setattr(ctx, "device", 1)
        with pytest.raises(AssertionError, match="not on the context's device"):
            ctx.wcc_rows_keep(d, x, codes, steps)
    ctx.wcc_rows_keep(d, x, codes, steps)
    assert int(codes[0, 0]) == 64
