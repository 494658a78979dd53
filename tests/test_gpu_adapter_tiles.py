"""The projection with adapters in whole 256 x 256 tiles, the last of which are moved back over others (needs an MI355X).  Tolerances
as in test_gpu_adapter.py."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import adapter_backward
from tests.test_gpu_adapter import backward, inputs, near

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
