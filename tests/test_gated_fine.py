"""The gated block's gradients in bf16 with dg and du in 16 bits where the caller asks for it (``TRAIN_FINE``), however many they are."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import ACTS, act
from tests.head_util import TYPES, rows_of
from tests.test_gpu_gated_exact import FEW, definition, inputs, kept_buffers


def test_workspace():
    """Room for second parts of dg and du; none for fp32, and none more where they have them anyway."""
    def room(rows, t, train):
        return wcc.gated_workspace_bytes(wcc.make_gated_desc(rows, 96, 640, t, train=train))
    assert room(5000, wcc.BF16, wcc.TRAIN_FINE) >= room(5000, wcc.BF16, True) + 5000 * 2 * 640 * 2
    assert room(5000, wcc.F32, wcc.TRAIN_FINE) == room(5000, wcc.F32, True)
    assert room(100, wcc.BF16, wcc.TRAIN_FINE) == room(100, wcc.BF16, True)


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def backward(ctx, d, args, dy, t, pad=0, shift=0):
    dx = rows_of(torch.full((d.rows, d.C_in), 9.0), TYPES[t], pad, shift)
    dw = [torch.full((d.C_out, d.C_in), 9.0, dtype=TYPES[t], device="cuda") for _ in range(2)]
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_gated_backward(d, *args, dy, dx, *dw)
    torch.cuda.synchronize()
    return {"dx": dx, "dw_gate": dw[0], "dw_up": dw[1]}


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(64, 320, 4000, 0, 0), (20, 200, 7000, 8, 0), (1500, 60, 90, 0, 0), (129, 7744, 1100, 0, 0), (3000, 100, 700, 0, 0),
                                  (600, 1024, 1030, 0, 3), (777, 1000, 1537, 3, 0), (4096, 512, 1024, 0, 0), (8192, 1024, 2048, 0, 0)],
                         ids=lambda s: "x".join(map(str, s)))
def test_whole_numbers(ctx, size):
    """dg and du of 15 bits, without an activation: exact but for one rounding of each result."""
    rows, ci, co, pad, shift = size
    assert rows * co >= FEW
    x, wg, wu, dy = inputs(rows, ci, co, sum(size), large=True)
    want, _, dg, du = definition(x, wg, wu, dy)
    rounded = dg.bfloat16().double().t() @ x.cuda().double()  # (8 bits would show)
    assert not torch.equal(rounded.bfloat16(), want["dw_gate"].bfloat16())
    x, dy = (rows_of(v, torch.bfloat16, pad, shift) for v in (x, dy))
    wg, wu = wg.bfloat16().cuda(), wu.bfloat16().cuda()
    d = wcc.make_gated_desc(rows, ci, co, wcc.BF16, wcc.ACT_NONE, wcc.TRAIN_FINE, ldx=ci + pad, ldy=co + pad)
    ctx.ensure_workspace(d)
    xk, gk = kept_buffers(rows, width=ci), kept_buffers(2, rows, width=co)
    y = rows_of(torch.zeros((rows, co)), torch.bfloat16, pad, shift)
    ctx.wcc_rows_keep(wcc.make_rows_desc(rows, ci, wcc.BF16, ld=ci + pad), x, *xk)
    ctx.wcc_gated_forward(d, x, wg, wu, y, *gk)
    assert torch.equal(y, want["y"].bfloat16())
    for way, args in (("x", (x, None, None, wg, wu, None, None)), ("x in 8 bits", (None, *xk, wg, wu, None, None)),
                      ("all in 8 bits", (None, *xk, wg, wu, *gk))):
        for k, v in backward(ctx, d, args, dy, "bf16", pad, shift).items():
            assert torch.equal(v, want[k].bfloat16()), (way, k)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("size", [(3000, 160, 600), (1156, 1024, 520), (60, 512, 3000)], ids=str)
def test_errors_are_those_of_one_rounding(ctx, name, size):
    """The whole gradient's distance from its definition is that of rounding it once (dg and du's 2^-17 and fp32's sums are below a hundredth of
    it; bf16's silu and gelu are off by 2^-22 and less); with dg and du in 8 bits it is 1.4 times as far."""
    rows, ci, co = size
    gen = torch.Generator().manual_seed(sum(size))
    x, dy = (torch.randn((rows, n), generator=gen).bfloat16().cuda() for n in (ci, co))
    wg, wu = ((torch.randn((co, ci), generator=gen) / math.sqrt(ci)).bfloat16().cuda() for _ in range(2))
    xd, gd, ud, top = (v.double() for v in (x, wg, wu, dy))
    g, u = xd @ gd.t(), xd @ ud.t()
    value, slope = act(g, name)
    dg, du = top * u * slope, top * value
    want = {"dx": dg @ gd + du @ ud, "dw_gate": dg.t() @ xd, "dw_up": du.t() @ xd}
    d = wcc.make_gated_desc(rows, ci, co, wcc.BF16, ACTS[name], wcc.TRAIN_FINE)
    for k, v in backward(ctx, d, (x, None, None, wg, wu, None, None), dy, "bf16").items():
        off, once = (v.double() - want[k]).norm(), (want[k].bfloat16().double() - want[k]).norm()
        assert float(off / once) < 1.02, (k, float(off / once))


@pytest.mark.gpu
def test_fp32_is_as_it_was(ctx):
    x, wg, wu, dy = (v.cuda() for v in inputs(300, 96, 640, 1))
    got = [backward(ctx, wcc.make_gated_desc(300, 96, 640, wcc.F32, train=train), (x, None, None, wg, wu, None, None), dy, "f32")
           for train in (True, wcc.TRAIN_FINE)]
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])
