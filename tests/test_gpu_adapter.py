"""wcc_adapter_forward and wcc_adapter_backward against their definitions in 64 bits and against differences (needs an MI355X).

An fp32 sum of n products is off by at most (n + 64) 2^-24 of the sum of their magnitudes, in any order and with the partial sums of
64 workgroups joined at the end.  The thin products carry that of their first factor through the second, and lose 2^-16 of a line's
value to the 16 bits that bf16 matrices meet it with (dA and dB keep all 24).  bf16 results are rounded once more, by 2^-8."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, adapter_backward, adapter_forward, around, rows_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def inputs(rows, ci, co, n, r, t, seed, pad=0, shift=0, ranks=True, order="mixed"):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[t]
    of_row = torch.randint(-1, n, (rows,), generator=gen)
    if order == "runs":
        of_row = of_row.sort().values
    if rows > 3:
        of_row[rows // 2] = n + 3  # outside: none
    rank = torch.randint(0, r + 1, (max(n, 1),), generator=gen)[:n]
    a = torch.randn((n, r, ci), generator=gen) / math.sqrt(ci)
    b = torch.randn((n, co, r), generator=gen) / math.sqrt(r)
    x = rows_of(torch.randn((rows, ci), generator=gen), dt, pad, shift)
    dy = rows_of(torch.randn((rows, co), generator=gen), dt, pad, shift)
    w = (torch.randn((co, ci), generator=gen) / math.sqrt(ci)).to(dt).cuda()
    a, b = a.to(dt).cuda(), b.to(dt).cuda()
    if ranks:  # lines past an adapter's rank hold anything
        for i in range(n):
            a[i, int(rank[i]):] = math.nan
            b[i, :, int(rank[i]):] = math.nan
    scale = (0.5 + torch.rand(n, generator=gen)).cuda()
    return x, w, of_row.to(torch.int32).cuda(), a, b, rank.to(torch.int32).cuda() if ranks else None, scale if ranks else None, dy


def desc_of(x, y, n, r):
    rows, ci = x.shape
    return wcc.make_adapter_desc(rows, ci, y.shape[1], n, r, wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32,
                                 ldx=x.stride(0) if rows > 1 else ci, ldy=y.stride(0) if rows > 1 else y.shape[1])


def forward(ctx, x, w, of_row, a, b, ranks, scale, pad=0, shift=0):
    y = rows_of(torch.full((x.shape[0], w.shape[0]), 9.0), x.dtype, pad, shift)
    d = desc_of(x, y, a.shape[0], a.shape[1])
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)  # whatever an earlier call left: here NaN
    ctx.wcc_adapter_forward(d, x, w, of_row, a, b, ranks, scale, y)
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(y)).all())
    return y


def backward(ctx, x, w, of_row, a, b, ranks, scale, dy, pad=0, shift=0, want=("dx", "da", "db")):
    dx = rows_of(torch.full(tuple(x.shape), 9.0), x.dtype, pad, shift)
    out = {"dx": dx, "da": torch.full(tuple(a.shape), 9.0, device="cuda"), "db": torch.full(tuple(b.shape), 9.0, device="cuda")}
    d = desc_of(x, dy, a.shape[0], a.shape[1])
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_adapter_backward(d, x, w, of_row, a, b, ranks, scale, dy, *[out[k] if k in want else None for k in ("dx", "da", "db")])
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(dx)).all())
    return out


def near(got, want, main, low, n_main, n_low, narrow):
    """n_main, n_low: products in a sum with W, and in the two thin ones together; narrow: the result's and the lines' type."""
    tol = (n_main + 64) * U * main + (n_low + 128) * U * low + 1e-30
    if narrow:
        tol = tol + 2.0 ** -16 * low + 2.0 ** -8 * 1.001 * (want.abs() + tol)
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


SIZES = [  # rows, C_in, C_out, adapters, rank, padding, shift
    (1, 1, 1, 1, 1, 0, 0), (1, 64, 64, 2, 4, 0, 0), (2, 3, 5, 1, 2, 1, 1), (1, 2048, 520, 3, 16, 0, 0), (7, 129, 63, 3, 5, 0, 3),
    (16, 256, 128, 4, 8, 8, 0), (17, 512, 272, 20, 16, 0, 0), (33, 1000, 137, 5, 24, 3, 1), (64, 320, 640, 2, 64, 0, 0),
    (65, 64, 257, 2, 128, 0, 0), (100, 72, 96, 7, 33, 8, 8), (130, 512, 384, 3, 16, 0, 0), (257, 200, 300, 2, 8, 0, 0), (300, 256, 520, 40, 12, 8, 0),
    (520, 640, 264, 3, 32, 0, 0), (600, 96, 48, 1, 1, 0, 1),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["mixed", "runs"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(ctx, t, order, size):
    rows, ci, co, n, r, pad, shift = size
    v = inputs(rows, ci, co, n, r, t, sum(size), pad, shift, order=order)
    y = forward(ctx, *v[:7], pad=pad, shift=shift)
    near(y, *adapter_forward(*v[:7]), ci, ci + r, t == "bf16")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["mixed", "runs"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(ctx, t, order, size):
    rows, ci, co, n, r, pad, shift = size
    v = inputs(rows, ci, co, n, r, t, sum(size) + 1, pad, shift, order=order)
    got, want = backward(ctx, *v, pad=pad, shift=shift), adapter_backward(*v)
    near(got["dx"], *want["dx"], co, co + r, t == "bf16")
    near(got["da"], *want["da"], 0, co + rows, False)
    near(got["db"], *want["db"], 0, ci + rows, False)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_optional_parts(ctx, t):
    """No ranks and scales, no adapters at all, rows of which none has one, some of the gradients only."""
    v = inputs(70, 96, 160, 3, 8, t, 1, ranks=False)
    near(forward(ctx, *v[:7]), *adapter_forward(*v[:7]), 96, 104, t == "bf16")
    want = adapter_backward(*v)
    for some in (("dx",), ("da",), ("db",), ("da", "db")):
        got = backward(ctx, *v, want=some)
        for k in ("dx", "da", "db"):
            if k not in some:
                assert bool((got[k] == 9).all())
        if "dx" in some:
            near(got["dx"], *want["dx"], 160, 168, t == "bf16")
        if "da" in some:
            near(got["da"], *want["da"], 0, 230, False)
        if "db" in some:
            near(got["db"], *want["db"], 0, 166, False)
    none = torch.full_like(v[2], -1)
    bare = adapter_forward(v[0], v[1], none, *v[3:7])
    assert torch.equal(forward(ctx, v[0], v[1], none, *v[3:7]), forward(ctx, v[0], v[1], None, *v[3:7]))
    near(forward(ctx, v[0], v[1], none, *v[3:7]), *bare, 96, 104, t == "bf16")
    got = backward(ctx, v[0], v[1], none, *v[3:])
    assert not bool(got["da"].any()) and not bool(got["db"].any())
    d = wcc.make_adapter_desc(70, 96, 160, 0, 0, wcc.BF16 if t == "bf16" else wcc.F32)
    y = torch.empty((70, 160), dtype=TYPES[t], device="cuda")
    ctx.ensure_workspace(d)
    ctx.wcc_adapter_forward(d, v[0], v[1], None, None, None, None, None, y)
    near(y, *bare, 96, 104, t == "bf16")


def test_no_rows(ctx):
    x, y = torch.empty((0, 64), device="cuda"), torch.empty((0, 32), device="cuda")
    w, a, b = torch.ones((32, 64), device="cuda"), torch.ones((2, 4, 64), device="cuda"), torch.ones((2, 32, 4), device="cuda")
    d = wcc.make_adapter_desc(0, 64, 32, 2, 4, wcc.F32)
    ctx.ensure_workspace(d)
    of_row = torch.empty(0, dtype=torch.int32, device="cuda")
    ctx.wcc_adapter_forward(d, x, w, of_row, a, b, None, None, y)
    da, db = torch.ones((2, 4, 64), device="cuda"), torch.ones((2, 32, 4), device="cuda")
    ctx.wcc_adapter_backward(d, x, w, of_row, a, b, None, None, y, x, da, db)
    assert not bool(da.any()) and not bool(db.any())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 2048, 256, 2, 8), (40, 1024, 512, 9, 16), (300, 512, 512, 4, 16)], ids=lambda s: "x".join(map(str, s)))
def test_equal_calls_give_equal_bits(ctx, t, size):
    v = inputs(*size, t, 5)
    y, g = forward(ctx, *v[:7]), backward(ctx, *v)
    for _ in range(3):
        assert torch.equal(y, forward(ctx, *v[:7]))
        again = backward(ctx, *v)
        assert all(torch.equal(g[k], again[k]) for k in g)


def test_gradients_against_differences(ctx):
    """Of sum(dy y), which is linear in x and in each of A and B: differences of the 64-bit definition are exact but for their
    rounding (1e-9 here), so what is compared is the gradients' own error, 2e-5 of the magnitudes that add up to them."""
    rows, ci, co, n, r = 5, 12, 9, 2, 3
    v = list(inputs(rows, ci, co, n, r, "f32", 3, ranks=False))
    v[2] = torch.tensor([0, 1, -1, 1, 0], dtype=torch.int32).cuda()
    got = backward(ctx, *v)
    dy = v[7].double().cpu()

    def value(k, at, h):
        u = [x.double().cpu() if torch.is_tensor(x) and x.is_floating_point() else x for x in v[:7]]
        u[k] = u[k].clone()
        u[k][at] += h
        return float((adapter_forward(*u)[0] * dy).sum())

    for k, name in ((0, "dx"), (3, "da"), (4, "db")):
        g = got[name].double().cpu()
        for at in [tuple(i.tolist()) for i in torch.ones_like(g).nonzero()][::7]:
            diff = (value(k, at, 0.5) - value(k, at, -0.5))
            assert abs(float(g[at]) - diff) <= 2e-5 * (1 + abs(diff)), (name, at)


@pytest.mark.parametrize("rows", [3, 130])
def test_rows_beyond_32_bit_offsets(ctx, rows):
    """Rows of x and y so far apart that the last ones begin beyond 2^32 elements."""
    ci, co, n, r = 64, 72, 2, 8
    ld = ((1 << 32) // (rows - 1) + 77) // 8 * 8
    v = inputs(rows, ci, co, n, r, "bf16", 9)
    want = forward(ctx, *v[:7])
    x = torch.empty(ld * (rows - 1) + ci, dtype=torch.bfloat16, device="cuda").as_strided((rows, ci), (ld, 1))
    y = torch.empty(ld * (rows - 1) + co, dtype=torch.bfloat16, device="cuda").as_strided((rows, co), (ld, 1))
    x.copy_(v[0])
    d = wcc.make_adapter_desc(rows, ci, co, n, r, wcc.BF16, ldx=ld, ldy=ld)
    if ld >= 1 << 31:
        with pytest.raises(wcc.WccError):
            ctx.wcc_adapter_forward(d, x, *v[1:7], y)
        return
    ctx.ensure_workspace(d)
    ctx.wcc_adapter_forward(d, x, *v[1:7], y)
    assert torch.equal(y.contiguous(), want.contiguous())


@pytest.mark.parametrize("size", [(1, 2048, 256, 2, 8), (200, 512, 512, 4, 16)], ids=lambda s: "x".join(map(str, s)))
def test_in_a_graph_and_on_another_stream(ctx, size):
    x, w, of_row, a, b, ranks, scale, dy = inputs(*size, "bf16", 6)
    own = wcc.Context(0)
    y, dx = torch.zeros_like(dy), torch.zeros_like(x)
    da, db = torch.zeros(tuple(a.shape), device="cuda"), torch.zeros(tuple(b.shape), device="cuda")
    d = desc_of(x, y, a.shape[0], a.shape[1])
    own.ensure_workspace(d)

    def both():
        own.wcc_adapter_forward(d, x, w, of_row, a, b, ranks, scale, y)
        own.wcc_adapter_backward(d, x, w, of_row, a, b, ranks, scale, dy, dx, da, db)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    first = [v.clone() for v in (y, dx, da, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (0, 7, 8):
        if seed:
            x.copy_(torch.randn(tuple(x.shape), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y, dx, da, db)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (y, dx, da, db)))
        if not seed:
            assert all(torch.equal(p, q) for p, q in zip(got, first))
    own.close()


def test_refusals(ctx):
    import ctypes as C
    x, w, of_row, a, b, ranks, scale, dy = inputs(8, 64, 32, 2, 4, "f32", 2, ranks=False)
    y, dx = torch.zeros_like(dy), torch.zeros_like(x)
    L, h = wcc.lib(), ctx._h
    good = dict(rows=8, C_in=64, C_out=32, adapters=2, rank=4, dtype=wcc.F32)
    d = wcc.make_adapter_desc(**good)
    ctx.ensure_workspace(d)

    def status(desc, args, call=L.wcc_adapter_forward):
        return call(h, C.byref(desc), *[None if v is None else C.c_void_p(v if isinstance(v, int) else v.data_ptr()) for v in args], None)

    args = [x, w, of_row, a, b, None, None, y]
    for hole in (0, 1, 3, 4, 7):
        assert status(d, [None if i == hole else v for i, v in enumerate(args)]) == 1, hole
    assert status(d, [x.data_ptr() + 2] + args[1:]) == 8
    for bad, want in ((dict(C_in=0), 2), (dict(C_out=0), 2), (dict(rows=-1), 2), (dict(rank=0), 2), (dict(rank=129), 6), (dict(adapters=-1), 2),
                      (dict(dtype=wcc.I8), 3), (dict(ldx=63), 2), (dict(ldy=31), 2)):
        kw = dict(good)
        kw.update(bad)
        assert status(wcc.make_adapter_desc(**kw), args) == want, bad
    back = [x, w, of_row, a, b, None, None, dy, dx, None, None]
    for hole in (1, 3, 4, 7):
        assert status(d, [None if i == hole else v for i, v in enumerate(back)], L.wcc_adapter_backward) == 1, hole
    da = torch.zeros((2, 4, 64), device="cuda")
    assert status(d, [None] + back[1:9] + [da, None], L.wcc_adapter_backward) == 1  # dA needs x
    fresh = wcc.Context(0)
    with pytest.raises(wcc.WccError) as e:
        fresh.wcc_adapter_forward(d, x, w, of_row, a, b, None, None, y)
    assert e.value.status == 5
    fresh.close()
    torch.cuda.synchronize()
