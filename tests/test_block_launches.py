"""Group norm of as many groups as a descriptor may have: a launch has fewer than 2^32 threads, whatever the route."""
import pytest
import torch

from paper_2205_12268_amd import wcc


def test_workspace_of_the_most_groups():
    """2^23 workgroups of 512 threads would be no launch: such a batch goes by way of chunks, whose sums the workspace holds."""
    samples, C = 1 << 23, 257
    sums = samples * C * 16
    assert wcc.group_norm_workspace_bytes(wcc.make_group_norm_desc(samples, 1, C, 1, wcc.BF16)) >= 2 * sums
    assert wcc.group_norm_workspace_bytes(wcc.make_group_norm_desc(samples // 2, 1, C, 1, wcc.BF16)) < sums


@pytest.mark.gpu
def test_the_most_groups():
    """A row a sample, 257 channels in one group: the first and last rows from their definition, and sums over all of them."""
    samples, C, eps = 1 << 23, 257, 1e-5
    ctx = wcc.Context(0)
    x = torch.empty((samples, C), dtype=torch.bfloat16, device="cuda")
    x[:], x[:5], x[-5:] = torch.linspace(-2, 2, C).cuda(), torch.randn((5, C)).cuda(), torch.randn((5, C)).cuda()
    y, stats = torch.zeros_like(x), torch.empty((samples, 1, 2), device="cuda")
    d = wcc.make_group_norm_desc(samples, 1, C, 1, wcc.BF16, wcc.ACT_NONE, eps)
    ctx.ensure_workspace(d)
    ctx.wcc_group_norm_forward(d, x, None, None, None, y, stats)
    dx, dgamma, dbeta = torch.zeros_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    dy = torch.ones_like(x)
    dy[-5:] = torch.randn((5, C)).cuda()
    ctx.wcc_group_norm_backward(d, x, None, None, None, None, None, stats, dy, dx, dgamma, dbeta)
    torch.cuda.synchronize()
    step = 2.0 ** -8  # half a step of bf16, relative; fp32's loss is far below a hundredth of it at values of about 1
    for at in (slice(0, 6), slice(samples - 6, samples)):
        v, top = x[at].double(), dy[at].double()
        rstd = 1 / (v.var(dim=1, unbiased=False, keepdim=True) + eps).sqrt()
        xh = (v - v.mean(dim=1, keepdim=True)) * rstd
        assert bool(((y[at].double() - xh).abs() <= 1.01 * step * xh.abs() + 1e-5).all())
        want = rstd * (top - top.mean(dim=1, keepdim=True) - xh * (top * xh).mean(dim=1, keepdim=True))
        assert bool(((dx[at].double() - want).abs() <= 1.01 * step * want.abs() + 1e-5).all())
    assert torch.equal(y[5:-5:1000], y[5:6].expand_as(y[5:-5:1000])) and torch.equal(stats[5:-5:1000], stats[5:6].expand_as(stats[5:-5:1000]))
    want = (samples - 5) + dy[-5:].double().sum(dim=0)
    assert bool(((dbeta.double() - want).abs() <= 2.0 ** -23 * want).all())
    ctx.close()
    del x, y, dx, dy, stats
    torch.cuda.empty_cache()
