"""The operators of a block on rows as a program uses them together (needs an MI355X): a training step of the example's block operator by
operator, each from its 64-bit definition on what the one before it wrote; the block in front of the head."""
import math

import pytest
import torch

from paper_2205_12268_amd import head, wcc
from paper_2205_12268_amd.block import GatedBlock
from tests.block_util import NARROW, U, gated_backward, gated_forward, group_norm, kept, near

pytestmark = pytest.mark.gpu


def values(pair, width):
    codes, steps = pair
    return (codes.double() * torch.exp2(steps.double() - 127).repeat_interleave(32, dim=-1))[..., :width].cpu()


@pytest.mark.parametrize("counts", [None, [70, 31, 0]])
def test_a_step_operator_by_operator(counts):
    samples, pixels, channels, hidden, groups = 3, 70, 48, 136, 6
    rows = samples * pixels
    gen = torch.Generator().manual_seed(4)
    ctx = wcc.Context(0)
    b = GatedBlock(ctx, samples, pixels, channels, hidden, groups)
    b.masters["gamma"] += 0.2 * torch.randn(channels, generator=gen).cuda()
    b.masters["beta"] += 0.2 * torch.randn(channels, generator=gen).cuda()
    x = torch.randn((rows, channels), generator=gen).bfloat16().cuda()
    dout = torch.randn((rows, channels), generator=gen).bfloat16().cuda()
    counts = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    there = torch.cat([torch.arange(pixels) < (pixels if counts is None else int(counts[i])) for i in range(samples)])
    out = b.forward(x, counts).clone()
    dx = b.backward(dout, counts).clone()
    torch.cuda.synchronize()
    m = b.masters
    # forward
    want = group_norm(x, samples, groups, m["gamma"], m["beta"], counts, 1e-5, "silu")
    near(b.n[there.cuda()], tuple(v[there] for v in want["y"]), True, "n")
    assert not bool(b.n[~there.cuda()].any())
    codes, steps, n = kept(b.n)
    assert torch.equal(b.n_kept[0].cpu(), codes) and torch.equal(b.n_kept[1].cpu(), steps)
    near(b.h, gated_forward(b.n, b.w_gate, b.w_up, "silu")["y"], True, "h")
    h, w = b.h.double().cpu(), b.w_down.double().cpu()
    y = h @ w.t()
    tol = (hidden + 64) * U * (h.abs() @ w.abs().t())
    tol = tol + NARROW * 1.01 * (y.abs() + tol)  # (the projection's own rounding, then that of the sum)
    near(out, (y + x.double().cpu(), tol), True, "out")
    # backward
    d = dout.double().cpu()
    near(b.dh, (d @ w, (channels + 64) * U * (d.abs() @ w.abs())), True, "dh")
    gu = values(b.h_kept, hidden)
    want = gated_backward(n, b.w_gate, b.w_up, "silu", b.dh, True, (gu[0], gu[1]))
    for k, got in (("dx", b.dn), ("dw_gate", b.grads["w_gate"]), ("dw_up", b.grads["w_up"])):
        near(got, want[k], True, k)
    xk = values(b.x_kept, channels)
    assert torch.equal(xk[there], kept(x)[2][there])
    xk[~there] = 0
    want = group_norm(x, samples, groups, m["gamma"], m["beta"], counts, 1e-5, "silu", b.dn, xk)
    value, tol = (v[there] for v in want["dx"])
    tol = tol + NARROW * 1.01 * (value.abs() + tol)
    near(dx[there.cuda()], (value + d[there], tol), True, "dx of the block")
    assert torch.equal(dx[~there.cuda()], dout[~there.cuda()])
    near(b.grads["gamma"], want["dgamma"], False, "dgamma")
    near(b.grads["beta"], want["dbeta"], False, "dbeta")
    ctx.close()


def test_the_block_in_front_of_the_head():
    losses, answers, _ = head.demo(steps=4, side=16, say=lambda _: None, with_block=True)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
    assert all(bool(torch.isfinite(a).all()) for a in answers)


def test_steps_in_a_graph():
    """Forward and backward captured together, replayed over other inputs: the eager step's bits."""
    ctx = wcc.Context(0)
    b = GatedBlock(ctx, 2, 64, 32, 64, 4)
    x, dout = (torch.randn((128, 32), device="cuda").bfloat16() for _ in range(2))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        b.forward(x)
        b.backward(dout)
    for seed in range(3):
        gen = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn((128, 32), generator=gen))
        dout.copy_(torch.randn((128, 32), generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        first = [v.clone() for v in (b.out, b.dx, *b.grads.values())]
        b.forward(x)
        b.backward(dout)
        torch.cuda.synchronize()
        for u, v in zip(first, (b.out, b.dx, *b.grads.values())):
            assert torch.equal(u, v)
    ctx.close()
