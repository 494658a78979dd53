"""One step of the example's tuning, each operator on what the one before it wrote, with the operators' own tolerances (needs an MI355X)."""
import pytest
import torch

from paper_2205_12268_amd import head, wcc
from tests.head_util import adapter_backward, adapter_forward, distill
from tests.test_gpu_adapter import near
from tests.test_gpu_distill import TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,channels,classes,rank", [(150, 64, 200, 4), (40, 96, 333, 8), (700, 72, 1000, 16)])
def test_a_step_operator_by_operator(rows, channels, classes, rank):
    gen = torch.Generator().manual_seed(rows)
    n, K, tau = 3, 7, 1.5
    x = torch.randn((rows, channels), generator=gen).bfloat16().cuda()
    w = (torch.randn((classes, channels), generator=gen) / 8).bfloat16().cuda()
    of_row = torch.randint(-1, n, (rows,), generator=gen, dtype=torch.int32).cuda()
    t_idx = torch.stack([torch.randperm(classes, generator=gen)[:K] for _ in range(rows)]).int().cuda()
    t_logit = (3 + torch.randn((rows, K), generator=gen)).cuda()
    ctx = wcc.Context(0)
    h = head.AdaptedHead(ctx, w, n, rank, rows, K, tau)
    h.a *= torch.tensor([1.0, 0.1, 10.0]).cuda()[:, None, None]  # adapters of unlike sizes: a factor missing in one shows
    h.b += 0.1 * torch.randn(h.b.shape, generator=gen).cuda() * torch.tensor([1.0, 0.01, 3.0]).cuda()[:, None, None]
    h._copies()
    a16, b16 = h.a16.clone(), h.b16.clone()
    y = h.project(x, of_row, h.logits).clone()
    near(y, *adapter_forward(x, w, of_row, a16, b16, None, None), channels, channels + rank, True)
    loss = h.step(x, of_row, t_idx, t_logit, 0.0).cpu().double()
    want_loss, _, grad, size = distill(y, t_idx, t_logit, tau, h.weight.cpu())
    assert bool(((loss - want_loss).abs() <= TOL * size).all())
    dy = h.logits  # (the logits' gradient has taken their place)
    q_mass = torch.zeros_like(grad).scatter_add_(1, t_idx.cpu().long(), torch.softmax(t_logit.cpu().double() / tau, 1))
    tol = 2 * TOL * (grad.abs() + 2 * tau / rows * q_mass) + 2.0 ** -8 * 1.001 * grad.abs() + 1e-30
    assert bool(((dy.double().cpu() - grad).abs() <= tol).all())
    want = adapter_backward(x, w, of_row, a16, b16, None, None, dy)
    near(h.da, *want["da"], 0, classes + rows, False)
    near(h.db, *want["db"], 0, channels + rows, False)
    ctx.close()
