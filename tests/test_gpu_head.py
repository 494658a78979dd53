"""The operators of a model's head together (needs an MI355X): adapters tuned by distillation on a WCC layer's maps, and the
answers afterwards."""
import pytest
import torch

from paper_2205_12268_amd import head, wcc
from tests.head_util import adapter_backward, adapter_forward, distill

pytestmark = pytest.mark.gpu


def test_tuning_brings_the_loss_down():
    losses, answers, _ = head.demo(steps=30, say=lambda _: None)
    assert losses[-1] < 0.9 * losses[0] and all(b < a for a, b in zip(losses, losses[1:]))
    logprob, entropy, best, best_logprob = answers
    assert bool((logprob <= best_logprob[:, 0] + 1e-6).all()) and bool((entropy > 0).all())
    assert bool((best_logprob[:, :-1] >= best_logprob[:, 1:]).all())


def test_one_step_is_the_formulas():
    """A whole step from its 64-bit formulas: logits rounded to bf16, their gradient to bf16, then dA and dB."""
    gen = torch.Generator().manual_seed(3)
    rows, channels, classes, n, rank, K = 150, 64, 200, 3, 4, 7
    x = torch.randn((rows, channels), generator=gen).bfloat16().cuda()
    w = (torch.randn((classes, channels), generator=gen) / 8).bfloat16().cuda()
    of_row = torch.randint(-1, n, (rows,), generator=gen, dtype=torch.int32).cuda()
    t_idx = torch.stack([torch.randperm(classes, generator=gen)[:K] for _ in range(rows)]).int().cuda()
    t_logit = (3 + torch.randn((rows, K), generator=gen)).cuda()
    ctx = wcc.Context(0)
    h = head.AdaptedHead(ctx, w, n, rank, rows, K, 1.5)
    h.b += 0.1 * torch.randn(h.b.shape, generator=gen).cuda()
    h._copies()
    a16, b16 = h.a16.clone(), h.b16.clone()
    loss = h.step(x, of_row, t_idx, t_logit, 0.0).clone()
    y = adapter_forward(x, w, of_row, a16, b16, None, None)[0].bfloat16()
    want_loss, _, grad, size = distill(y, t_idx, t_logit, 1.5, h.weight.cpu())
    # (a logit that rounds the other way moves the loss by 2^-8 of itself at most, against the gradient's sum of 2 tau)
    assert bool(((loss.cpu().double() - want_loss).abs() <= 3.0 * 2.0 ** -8 * float(y.abs().max())).all())
    want = adapter_backward(x, w, of_row, a16, b16, None, None, grad.bfloat16())
    for got, (v, _, mag) in ((h.da, want["da"]), (h.db, want["db"])):
        assert float((got.double().cpu() - v).abs().max()) <= 2.0 ** -5 * float(mag.max())
    ctx.close()
