"""The operators of a block on rows where offsets pass 32 bits (needs an MI355X): rows, weights and codes of more than 2^31 elements.  Whole
numbers, as in test_gpu_gated_exact, so that every result is exact but for one rounding of bf16."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import CODE, TYPES
from tests.test_gpu_gated_exact import kept_buffers

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()
    torch.cuda.empty_cache()


def sparse(rows, width, one_in, t, seed):
    """-1, 0 and 1, one of `one_in` not 0, made some rows at a time."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty((rows, width), dtype=TYPES[t], device="cuda")
    for part in out.split(max((1 << 27) // width, 1)):
        r = torch.randint(0, 2 * one_in, part.shape, generator=gen, dtype=torch.uint8, device="cuda")
        part.copy_((r == 0).to(torch.int8) - (r == 1).to(torch.int8))
    return out


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_many_rows(ctx, t):
    rows, ci, co = (1 << 21) + 5, 8, 1056
    assert rows * co > 1 << 31
    x, wg, wu, dy = sparse(rows, ci, 2, t, 1), sparse(co, ci, 2, t, 2), sparse(co, ci, 2, t, 3), sparse(rows, co, 16, t, 4)
    y, (codes, steps), xk = torch.zeros_like(dy), kept_buffers(2, rows, width=co), kept_buffers(rows, width=ci)
    d = wcc.make_gated_desc(rows, ci, co, CODE[t], wcc.ACT_NONE, True)
    ctx.ensure_workspace(d)
    ctx.wcc_gated_forward(d, x, wg, wu, y, codes, steps)
    ctx.wcc_rows_keep(wcc.make_rows_desc(rows, ci, CODE[t]), x, *xk)
    got = {}
    for way, args in (("from x", (x, None, None, wg, wu, None, None)), ("from codes", (None, *xk, wg, wu, codes, steps))):
        got[way] = torch.zeros_like(x), torch.zeros_like(wg), torch.zeros_like(wu)
        ctx.wcc_gated_backward(d, *args, dy, *got[way])
    dwg, dwu = (torch.zeros((co, ci), dtype=torch.float64, device="cuda") for _ in range(2))
    gd, ud = wg.double(), wu.double()
    for i in range(0, rows, 1 << 18):
        at = slice(i, min(i + (1 << 18), rows))
        v, top = x[at].double(), dy[at].double()
        g, u = v @ gd.t(), v @ ud.t()
        assert torch.equal(y[at], (g * u).to(y.dtype)), i
        dg, du = top * u, top * g
        dx = (dg @ gd + du @ ud).to(y.dtype)
        assert all(torch.equal(got[way][0][at], dx) for way in got), i
        dwg += dg.t() @ v
        dwu += du.t() @ v
    assert float(dwg.abs().max()) < 1 << 24  # (and its sums of magnitudes: 2^21 / 16 products of 8 at most)
    for way in got:
        assert torch.equal(got[way][1], dwg.to(y.dtype)) and torch.equal(got[way][2], dwu.to(y.dtype)), way


@pytest.mark.parametrize("rows", [3, 70])
def test_large_weights(ctx, rows):
    ci, co = 65544, 32776
    assert ci * co > 1 << 31
    x, dy = sparse(rows, ci, 2, "bf16", 1), sparse(rows, co, 2, "bf16", 2)
    wg, wu = sparse(co, ci, 120, "bf16", 3), sparse(co, ci, 120, "bf16", 4)
    y, (codes, steps) = torch.zeros_like(dy), kept_buffers(2, rows, width=co)
    dx, dwg, dwu = torch.zeros_like(x), torch.zeros_like(wg), torch.zeros_like(wu)
    d = wcc.make_gated_desc(rows, ci, co, wcc.BF16, wcc.ACT_NONE, True)
    ctx.ensure_workspace(d)
    ctx.wcc_gated_forward(d, x, wg, wu, y, codes, steps)
    ctx.wcc_gated_backward(d, x, None, None, wg, wu, None, None, dy, dx, dwg, dwu)
    want, v = torch.zeros((rows, ci), dtype=torch.float64, device="cuda"), x.double()
    for i in range(0, co, 1 << 11):
        at = slice(i, min(i + (1 << 11), co))
        a, b = wg[at].double(), wu[at].double()
        g, u = v @ a.t(), v @ b.t()
        assert float(g.abs().max()) <= 127 and float(u.abs().max()) <= 127
        assert torch.equal(y[:, at], (g * u).bfloat16()), i
        dg, du = dy[:, at].double() * u, dy[:, at].double() * g
        want += dg @ a + du @ b
        assert torch.equal(dwg[at], (dg.t() @ v).bfloat16()) and torch.equal(dwu[at], (du.t() @ v).bfloat16()), i
    assert torch.equal(dx, want.bfloat16())
    first = dwg.clone()
    dwg.zero_(), dx.zero_()
    ctx.wcc_gated_backward(d, x, None, None, wg, wu, codes, steps, dy, dx, dwg)
    assert torch.equal(dwg, first) and torch.equal(dx, want.bfloat16())


def test_norm_from_codes(ctx):
    """A sample of more than 2^31 values in 8 bits: its last pixels, and sums over all of them."""
    pixels, C, eps = (1 << 25) + 3, 65, 1e-5
    x = torch.full((pixels, C), 1.0, dtype=torch.bfloat16, device="cuda")
    x[::2] = -1.0  # (one pixel more at -1 than at 1)
    y, (codes, steps) = torch.zeros_like(x), kept_buffers(pixels, width=C)
    d = wcc.make_group_norm_desc(1, pixels, C, 1, wcc.BF16, wcc.ACT_NONE, eps)
    ctx.ensure_workspace(d)
    stats = torch.empty((1, 1, 2), device="cuda")
    ctx.wcc_group_norm_forward(d, x, None, None, None, y, stats, codes, steps)
    assert bool((y == x).all())  # (mean -3e-8, variance 1: bf16 has nothing of the difference)
    assert torch.equal(codes[-3:, :C], (64 * x[-3:]).to(torch.int8)) and bool((steps == 127 - 6).all())  # (1 is 64 steps of 2^-6)
    dx, dgamma, dbeta = torch.zeros_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    y[-1] = 3.0
    ctx.wcc_group_norm_backward(d, None, codes, steps, None, None, None, stats, y, dx, dgamma, dbeta)
    assert float(dx[-1, 0]) == pytest.approx(4.0, rel=2.0 ** -8) and float(dbeta[7]) == pytest.approx(3.0, abs=1e-3)
    assert float(dgamma[64]) == pytest.approx((pixels - 4) / math.sqrt(1 + eps), rel=1e-6)  # (xh is x rstd)
