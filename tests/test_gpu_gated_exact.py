"""wcc_gated_forward and wcc_gated_backward on whole numbers (needs an MI355X), bit for bit.

Without an activation all of y = g u, dg = dy u, du = dy g and the gradients are whole numbers.  Here each sum of magnitudes is below 2^24,
so that fp32 sums are exact in any order, however k is cut and joined; projections are 127 at most, so that 8 bits hold them, and
dg and du have as many bits as they are held in (8, or 16 where they are in two parts).  What is left is one rounding of each bf16 result,
which is the same here: a k, a row or a range of either that is lost or taken twice shows, however long the sum is."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import CODE, TYPES, around, rows_of

pytestmark = pytest.mark.gpu
FEW = 1 << 17  # fewer values than this of dg and of du are held in two parts


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def whole(gen, density, *shape):
    """-1, 0 and 1"""
    v = torch.randint(0, 2, shape, generator=gen, dtype=torch.int8) * 2 - 1
    return (v * (torch.rand(shape, generator=gen) < density)).float()


def inputs(rows, ci, co, seed, large=False):
    """x, both weights, dy in fp32 on the CPU; large: dy up to 255."""
    gen = torch.Generator().manual_seed(seed)
    x, (wg, wu) = whole(gen, 2 / 3, rows, ci), whole(gen, min(2 / 3, 600 / ci), 2, co, ci)  # (projections of about 20 at most)
    dy = torch.randint(-255, 256, (rows, co), generator=gen).float() if large else whole(gen, 0.5, rows, co)
    return x, wg, wu, dy


def definition(x, wg, wu, dy):
    """Results in 64 bits (on the GPU: long sums), after the conditions that make them exact."""
    x, wg, wu, dy = (v.cuda().double() for v in (x, wg, wu, dy))
    g, u = x @ wg.t(), x @ wu.t()
    assert float(g.abs().max()) <= 127 and float(u.abs().max()) <= 127
    dg, du = dy * u, dy * g
    assert float((dg.abs() @ wg.abs() + du.abs() @ wu.abs()).max()) < 1 << 24
    assert float(torch.maximum((dg.abs().t() @ x.abs()).max(), (du.abs().t() @ x.abs()).max())) < 1 << 24
    want = {"y": g * u, "dx": dg @ wg + du @ wu, "dw_gate": dg.t() @ x, "dw_up": du.t() @ x}
    return want, torch.stack([g, u]), dg, du


def kept_buffers(*lead, width):
    room = wcc.kept_room(width)
    return (torch.full((*lead, room), 77, dtype=torch.int8, device="cuda"), torch.full((*lead, room // 32), 77, dtype=torch.uint8, device="cuda"))


def run(ctx, x, wg, wu, dy, pad=0, shift=0, some=("dx", "dw_gate", "dw_up")):
    """{way: {result}}: forward, and the gradients from x, from x in 8 bits, and from all in 8 bits."""
    rows, ci = x.shape
    co, t = wg.shape[0], x.dtype
    code = CODE["bf16" if t == torch.bfloat16 else "f32"]
    stride = lambda v: v.stride(0) if rows > 1 else v.shape[1]  # noqa: E731
    room = lambda width: rows_of(torch.full((rows, width), 9.0), t, pad, shift)  # noqa: E731
    y, (codes, steps) = room(co), kept_buffers(2, rows, width=co)
    d = wcc.make_gated_desc(rows, ci, co, code, wcc.ACT_NONE, True, ldx=stride(x), ldy=stride(y))
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_gated_forward(d, x, wg, wu, y, codes, steps)
    again = room(co)
    ctx.wcc_gated_forward(d, x, wg, wu, again)
    xk = kept_buffers(rows, width=ci)
    ctx.wcc_rows_keep(wcc.make_rows_desc(rows, ci, code, ld=stride(x)), x, *xk)
    out = {"forward": {"y": y}, "forward without codes": {"y": again}}
    for way, args in (("x", (x, None, None, wg, wu, None, None)), ("x in 8 bits", (None, *xk, wg, wu, None, None)),
                      ("all in 8 bits", (None, *xk, wg, wu, codes, steps))):
        got = {"dx": room(ci), "dw_gate": torch.full_like(wg, 9.0), "dw_up": torch.full_like(wg, 9.0)}
        ctx._ws.fill_(255)
        ctx.wcc_gated_backward(d, *args, dy, *[got[k] if k in some else None for k in ("dx", "dw_gate", "dw_up")])
        out[way] = {k: got[k] for k in some}
    torch.cuda.synchronize()
    assert all(bool(torch.isnan(around(v)).all()) for v in (y, again, *[out[w]["dx"] for w in out if "dx" in out[w]]))
    return out, (codes, steps)


def check(ctx, rows, ci, co, t, pad=0, shift=0, large=False, planted=True):
    x, wg, wu, dy = inputs(rows, ci, co, rows + ci + co, large)
    want, gu, dg, du = definition(x, wg, wu, dy)
    near = {k: v.to(TYPES[t]) for k, v in want.items()}
    if planted:  # a lost row, output or k (in the definition) would show
        xd, wgd = x.cuda().double(), wg.cuda().double()
        assert not torch.equal((want["dw_gate"] - dg[-1:].t() @ xd[-1:]).to(TYPES[t]), near["dw_gate"])
        assert not torch.equal((want["dx"] - dg[:, -1:] @ wgd[-1:]).to(TYPES[t]), near["dx"])
        assert not torch.equal(((gu[0] - xd[:, -1:] @ wgd[:, -1:].t()) * gu[1]).to(TYPES[t]), near["y"])
    x, dy = (rows_of(v, TYPES[t], pad, shift) for v in (x, dy))
    wg, wu = wg.to(TYPES[t]).cuda(), wu.to(TYPES[t]).cuda()
    got, (codes, steps) = run(ctx, x, wg, wu, dy, pad, shift)
    for i in (0, 1):
        back = codes[i].double() * torch.exp2(steps[i].double() - 127).repeat_interleave(32, dim=1)
        assert torch.equal(back[:, :co], gu[i]) and not bool(back[:, co:].any()), "codes"
    for way, results in got.items():
        for k, v in results.items():
            assert torch.equal(v, near[k]), (way, k, int((v != near[k]).sum()))
    for some in (("dx",), ("dw_gate",), ("dw_up",)):
        for way, results in run(ctx, x, wg, wu, dy, pad, shift, some)[0].items():
            for k, v in results.items():
                assert torch.equal(v, near[k]), (way, k, "by itself")


SIZES = [  # rows, C_in, C_out, padding, shift
    (3, 40, 17, 0, 0), (2, 33, 50, 1, 1), (7, 129, 63, 0, 3), (16, 256, 128, 8, 0), (33, 1000, 137, 3, 1), (64, 320, 640, 0, 0),
    (2, 7744, 512, 0, 0), (20, 5000, 72, 8, 0), (64, 4360, 33, 0, 0), (65, 64, 257, 0, 0), (130, 512, 384, 0, 0), (257, 200, 300, 0, 0),
    (520, 640, 264, 0, 0), (65, 4096, 520, 0, 0), (129, 2056, 513, 8, 0), (256, 2048, 256, 0, 0), (777, 1000, 1537, 3, 0), (700, 1001, 800, 0, 1),
    (600, 1024, 1030, 0, 3), (3500, 72, 1900, 0, 0), (3700, 3400, 40, 0, 0), (90, 8, 200000, 0, 0), (100, 64, 40000, 0, 0), (20011, 264, 72, 0, 0),
    (2000, 136, 1480, 0, 0), (1156, 160, 960, 0, 0), (66, 900, 640, 0, 0), (3000, 100, 700, 0, 0), (257, 7744, 512, 0, 0), (70, 3, 90000, 0, 0),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_whole_numbers(ctx, t, size):
    rows, ci, co, pad, shift = size
    check(ctx, rows, ci, co, t, pad, shift)


@pytest.mark.parametrize("size", [(1, 64, 64, 0, 0), (3, 40, 72, 0, 0), (16, 256, 128, 8, 0), (64, 320, 640, 0, 0), (65, 64, 257, 0, 0), (129, 2056, 513, 8, 0),
                                  (130, 512, 384, 0, 0), (257, 200, 300, 0, 0), (66, 900, 640, 0, 3), (1000, 4096, 130, 0, 0), (1900, 300, 68, 3, 0),
                                  (2, 7744, 512, 0, 0)], ids=lambda s: "x".join(map(str, s)))
def test_two_parts(ctx, size):
    """dg and du of 15 bits, in two parts of bf16."""
    rows, ci, co, pad, shift = size
    assert rows * co < FEW
    check(ctx, rows, ci, co, "bf16", pad, shift, large=True, planted=False)


@pytest.mark.parametrize("t,size", [("bf16", (4096, 2048, 5632)), ("bf16", (8192, 512, 1024)), ("bf16", (8192, 1024, 256)), ("f32", (4096, 512, 2048)),
                                    ("f32", (40000, 160, 960))], ids=str)
def test_large(ctx, t, size):
    """The largest tiles."""
    check(ctx, *size, t, planted=False)
