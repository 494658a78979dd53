"""Group norm with y in the place of x and dx in that of dy, on every route (needs an MI355X): the bits of the call with tensors of their
own.  Threads load whole vectors that reach over neighbours' channels and repeat rows of others, which may have been written by then."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.block_util import ACTS
from tests.head_util import CODE, around, rows_of
from tests.test_gpu_group_norm import EPS, backward, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


SIZES = [  # samples, pixels, C, groups, padding, shift, counts: held by registers; joined by the second pass; by a launch of their own
    (3, 40, 21, 7, 1, 1, [40, 0, 9]), (2, 100, 90, 9, 0, 0, None), (1, 5000, 20, 4, 0, 0, None), (2, 5000, 27, 3, 3, 1, [4999, 17]),
    (2, 4097, 363, 3, 0, 0, [4097, 2050]), (1, 3000, 1061, 1, 2, 1, None), (70, 300, 1030, 2, 0, 0, None), (1, 9000, 5, 5, 0, 3, None),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_in_place(ctx, t, size):
    samples, pixels, C, groups, pad, shift, counts = size
    x, gamma, beta, counts, dy = inputs(samples, pixels, C, t, sum(size[:4]) + 5, pad, shift, counts)
    n = [pixels] * samples if counts is None else counts.tolist()
    there = torch.cat([torch.arange(pixels) < k for k in n]).cuda()
    d = wcc.make_group_norm_desc(samples, pixels, C, groups, CODE[t], ACTS["gelu"], EPS, ldx=C + pad, ldy=C + pad)
    first = forward(ctx, x, samples, groups, "gelu", gamma, beta, counts, pad, shift)
    for keep in (False, True):
        z, stats = rows_of(x.clone(), x.dtype, pad, shift), torch.full_like(first["stats"], 9.0)
        codes, steps = (torch.full_like(first[k], 77) if keep else None for k in ("codes", "steps"))
        ctx._ws.fill_(255)
        ctx.wcc_group_norm_forward(d, z, gamma, beta, counts, z, stats, codes, steps)
        torch.cuda.synchronize()
        assert torch.equal(z[there], first["y"][there]) and torch.equal(z[~there], x[~there]) and bool(torch.isnan(around(z)).all())
        assert torch.equal(stats, first["stats"])
        assert not keep or (torch.equal(codes, first["codes"]) and torch.equal(steps, first["steps"]))
    for args in ((x, None), (None, (first["codes"], first["steps"]))):
        want = backward(ctx, args[0], args[1], samples, groups, "gelu", gamma, beta, counts, first["stats"], dy, pad, shift)
        g, dgamma, dbeta = rows_of(dy.clone(), dy.dtype, pad, shift), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ctx._ws.fill_(255)
        ctx.wcc_group_norm_backward(d, args[0], *(args[1] or (None, None)), gamma, beta, counts, first["stats"], g, g, dgamma, dbeta)
        torch.cuda.synchronize()
        assert torch.equal(g[there], want["dx"][there]) and torch.equal(g[~there], dy[~there]) and bool(torch.isnan(around(g)).all())
        assert torch.equal(dgamma, want["dgamma"]) and torch.equal(dbeta, want["dbeta"])
