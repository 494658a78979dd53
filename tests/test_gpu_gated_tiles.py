"""The gated block for many rows, on the routes that take tiles straight from memory: sizes on both sides of whole tiles, rows
and weights that have to be copied, ranges of k, the largest tiles (needs an MI355X).  Bounds as in test_gpu_gated."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import gated_backward, gated_forward, kept_on_gpu, near
from tests.test_gpu_gated import backward, forward, inputs, kept_near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


SIZES = [  # rows, C_in, C_out, padding, shift
    (65, 4096, 520, 0, 0), (300, 1024, 520, 0, 0), (129, 2056, 513, 8, 0), (256, 2048, 256, 0, 0), (777, 1000, 1537, 3, 0), (700, 1001, 800, 0, 1),
    (1024, 200, 704, 8, 8), (600, 1024, 1030, 0, 3), (3500, 72, 1900, 0, 0), (3700, 3400, 40, 0, 0), (90, 8, 200000, 0, 0), (100, 64, 40000, 0, 0),
    (20011, 264, 72, 0, 0), (2000, 136, 1480, 0, 0),
]


F32_SIZES = [(300, 1004, 130, 0, 0), (700, 52, 1000, 4, 4), (129, 2056, 513, 8, 0), (1156, 160, 960, 0, 0), (600, 400, 76, 0, 0), (66, 900, 640, 0, 0),
             (3000, 100, 700, 0, 0), (200, 2000, 1501, 0, 0), (700, 1001, 100, 0, 0), (400, 600, 300, 3, 1)]


@pytest.mark.parametrize("size", [("bf16", *s) for s in SIZES] + [("f32", *s) for s in F32_SIZES], ids=lambda s: "x".join(map(str, s)))
def test_both_directions(ctx, size):
    t, rows, ci, co, pad, shift = size
    narrow = t == "bf16"
    x, wg, wu, dy = inputs(rows, ci, co, t, sum(size[1:]), pad, shift)
    y, codes, steps = forward(ctx, x, wg, wu, "silu", pad, shift)
    want = gated_forward(x, wg, wu, "silu")
    near(y, want["y"], narrow)
    if rows * co < 3e6:
        kept_near(codes[0], steps[0], want["g"])
        kept_near(codes[1], steps[1], want["u"])
    assert torch.equal(forward(ctx, x, wg, wu, "silu", pad, shift, keep=False)[0], y)
    del want
    got, want = backward(ctx, x, None, wg, wu, "silu", dy, None, pad, shift), gated_backward(x, wg, wu, "silu", dy, narrow)
    for k in want:
        near(got[k], want[k], narrow, k)
    for some in (("dw_gate",), ("dw_up",)):
        assert torch.equal(backward(ctx, x, None, wg, wu, "silu", dy, None, pad, shift, want=some)[some[0]], got[some[0]])
    if rows * ci > 1e6:
        return
    *x_kept, values = kept_on_gpu(x)
    gu = [codes[i].double().cpu()[:, :co] * torch.exp2(steps[i].double().cpu() - 127).repeat_interleave(32, dim=1)[:, :co] for i in (0, 1)]
    got = backward(ctx, None, x_kept, wg, wu, "silu", dy, (codes, steps), pad, shift)
    want = gated_backward(values, wg, wu, "silu", dy, narrow, gu)
    for k in want:
        near(got[k], want[k], narrow, k + " from all in 8 bits")
    got, want = backward(ctx, None, x_kept, wg, wu, "silu", dy, None, pad, shift), gated_backward(values, wg, wu, "silu", dy, narrow)
    for k in want:
        near(got[k], want[k], narrow, k + " from x in 8 bits")


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(400, 1000, 700), (3500, 80, 1900)], ids=str)
def test_equal_calls_give_equal_bits(ctx, t, size):
    x, wg, wu, dy = inputs(*size, t, 3)
    first, second = (forward(ctx, x, wg, wu, "gelu") for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    first, second = (backward(ctx, x, None, wg, wu, "gelu", dy) for _ in range(2))
    assert all(torch.equal(first[k], second[k]) for k in first)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_row(ctx, t):
    """Infinities and NaN in a row of x, and in the last line of a weight beside the end of a tile."""
    x, wg, wu, dy = inputs(500, 1032, 600, t, 4)
    y, dx = forward(ctx, x, wg, wu, "silu")[0], backward(ctx, x, None, wg, wu, "silu", dy)["dx"]
    x[499, 1031] = float("nan")
    y2, dx2 = forward(ctx, x, wg, wu, "silu")[0], backward(ctx, x, None, wg, wu, "silu", dy)["dx"]
    assert torch.equal(y2[:499], y[:499]) and torch.equal(dx2[:499], dx[:499])
    assert bool(torch.isnan(y2[499]).all()) and bool(torch.isnan(dx2[499]).all())
    x, wg, wu, dy = inputs(500, 1032, 600, t, 4)
    wu[599] = float("inf")
    y2 = forward(ctx, x, wg, wu, "silu")[0]
    assert torch.equal(y2[:, :599], y[:, :599]) and not bool(torch.isfinite(y2[:, 599]).any())
