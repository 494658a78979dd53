"""Distillation where logits / temperature leave fp32's range or its precision (needs an MI355X)."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, distill, logits_like, rows_of
from tests.test_gpu_distill import TOL, check, run, teacher

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("t,tt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("V", [7, 600, 150000])
def test_a_teacher_below_the_range(ctx, t, tt, V):
    """Pairs whose logit / temperature lies below fp32's range are none: a row that has no others has loss 0 and gradient 0."""
    x = rows_of(logits_like(5, V, V), TYPES[t], pad=1)
    idx, z = teacher(5, V, 6, V, t=tt)
    z[1] = torch.finfo(TYPES[tt]).min
    z[2, 1:] = torch.finfo(TYPES[tt]).min
    z[3, :2] = -math.inf
    z[3, 2:] = torch.finfo(TYPES[tt]).min
    for mode in ("step", "two", "loss"):
        loss, _, grad = run(ctx, x, idx, z, 0.5, mode=mode, pad=1)
        assert float(loss[1]) == 0 and float(loss[3]) == 0
        if mode != "loss":
            assert not bool(grad[1].any()) and not bool(grad[3].any())
    masked = torch.where(z.double() * 2 < -torch.finfo(torch.float32).max, -math.inf, z.double()).to(z.dtype)  # what the definition sees
    loss, _, want, size = distill(x, idx, masked, 0.5)
    for mode in ("step", "two"):
        got_loss, _, grad = run(ctx, x, idx, z, 0.5, mode=mode, pad=1)
        assert bool(((got_loss - loss).abs() <= TOL * size).all())
        again = run(ctx, x, idx, masked, 0.5, mode=mode, pad=1)
        assert torch.equal(again[0], got_loss) and torch.equal(again[2].contiguous(), grad.contiguous())
    check(ctx, x, idx, masked, 0.5, pad=1)
