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


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [0.7, 1.5, 2.0, 3.0])
@pytest.mark.parametrize("V", [9, 700, 150001])
def test_the_gradient_beside_a_large_maximum(ctx, t, tau, V):
    """The gradient from a row's stats where m = largest / temperature is so large that fp32's steps beside it are wider than what
    exp() tells apart: rows of a mask's lowest value, of equal values, and with one far above the rest."""
    z = logits_like(9, V, V)
    z[0] = torch.finfo(TYPES[t]).min / 2  # (times 1 / 0.7 within the range)
    z[1] = -1e30
    z[2] = 3.3e9
    z[3] = 7.7e20
    z[4, V // 2] = 1.1e12
    z[5] = torch.where(torch.arange(V) % 2 == 0, 5.0e15, 4.0e15)
    z[6] = 2.0 ** 28 * tau - 2.0 ** 12 * tau * (1 + torch.arange(V) % 5)  # just below 2^28, steps of thousands
    z[7] = 1e7
    x = rows_of(z, TYPES[t], pad=3)
    idx, tz = teacher(9, V, min(V, 4), V)
    idx[:8] = -1  # (where p is 0 and q is not the loss is beyond any tolerance: one pair, at a largest logit)
    idx[:8, 0] = x[:8].argmax(dim=1).int()
    weight = torch.linspace(0.5, 2.0, 9).cuda()
    _, _, want, _ = distill(x, idx, tz, tau, weight.cpu())
    for mode in ("step", "two"):
        _, stats, grad = run(ctx, x, idx, tz, tau, weight, mode, pad=3)
        assert bool(torch.isfinite(stats).all()) and bool((stats[:, 1].abs() <= 50).all())
        scale = (tau * weight.cpu().double())[:, None]
        tol = 2 * TOL * (want.abs() + 2 * scale * (torch.zeros_like(want).scatter(1, idx.cpu().long().clamp(min=0), 1.0))) + 1e-30
        if t == "bf16":
            tol = tol + 2.0 ** -8 * 1.001 * want.abs()
        off = (grad.double().cpu() - want).abs()
        assert bool((off <= tol).all()), (mode, (off / tol).amax(dim=1))
