"""The projection with adapters in whole 256 x 256 tiles, the last of which are moved back over others (needs an MI355X).  Tolerances
as in test_gpu_adapter.py."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import adapter_backward
from tests.test_gpu_adapter import backward, forward, inputs, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("ci,co,pad", [(3529, 512, 0), (3524, 512, 4), (3582, 520, 1), (3535, 500, 0)])
def test_gradients_of_widths_between_chunks(ctx, ci, co, pad):
    """dx as wide as no whole chunks of 8: W is copied, and the last tile begins at a chunk of the copy."""
    rows, n, r = 4001, 3, 16
    v = inputs(rows, ci, co, n, r, "bf16", ci + co, pad, 0, order="runs")
    got, want = backward(ctx, *v, pad=pad), adapter_backward(*v)
    near(got["dx"], *want["dx"], co, co + r, True)
    near(got["da"], *want["da"], 0, co + rows, False)
    near(got["db"], *want["db"], 0, ci + rows, False)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("outs", [3528, 3531])
def test_outputs_of_two_tiles_are_stored_by_one(ctx, outs, bad):
    """The last tile of outputs covers some of the one before.  One element of an adapter that lies in the last one only, rank 40 (three
    steps, of which one is summed apart there): the outputs before keep the bits they have with a finite adapter, call for call."""
    rows, ci, n, r = 4001, 72, 4, 40
    v = list(inputs(rows, ci, outs, n, r, "bf16", 21, ranks=False, order="runs"))
    y = forward(ctx, *v[:7])
    v[4] = v[4].clone()
    v[4][1, outs - 200, 3] = bad
    last = (outs - 1) // 256 * 256  # where the last tile's own outputs begin
    first = forward(ctx, *v[:7])
    assert torch.equal(first[:, :last], y[:, :last])
    for _ in range(4):
        again = forward(ctx, *v[:7])
        assert torch.equal(again.contiguous().view(torch.int16), first.contiguous().view(torch.int16))
    v = list(inputs(rows, outs, 320, n, r, "bf16", 22, ranks=False, order="runs"))  # (dx as wide as y was; 3531: W is copied)
    g = backward(ctx, *v, want=("dx",))["dx"]
    v[3] = v[3].clone()
    v[3][1, 3, outs - 200] = bad
    first = backward(ctx, *v, want=("dx",))["dx"]
    assert torch.equal(first[:, :last], g[:, :last])
    for _ in range(4):
        again = backward(ctx, *v, want=("dx",))["dx"]
        assert torch.equal(again.contiguous().view(torch.int16), first.contiguous().view(torch.int16))
