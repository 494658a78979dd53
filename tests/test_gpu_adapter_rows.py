"""The projection with adapters at many rows, where whole tiles are taken (with and without the last ones moved back over others,
and in ranges of k), and what rows and adapters that are not finite do to the others (needs an MI355X).  Tolerances as in
test_gpu_adapter.py, of which they are."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import adapter_backward, adapter_forward
from tests.test_gpu_adapter import backward, forward, inputs, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


MANY = [  # type, rows, width, outputs, adapters, rank, padding, shift, order
    ("bf16", 4001, 200, 3528, 5, 16, 0, 0, "runs"), ("bf16", 4001, 328, 3528, 3, 40, 8, 8, "mixed"),
    ("bf16", 4001, 72, 3528, 2, 128, 0, 0, "runs"), ("f32", 2200, 72, 1800, 2, 128, 0, 0, "mixed"),
    ("bf16", 1500, 264, 2056, 30, 24, 0, 0, "mixed"), ("bf16", 1500, 136, 2051, 4, 128, 0, 0, "runs"),
    ("bf16", 2200, 75, 1801, 6, 8, 3, 1, "mixed"), ("f32", 2200, 72, 1800, 6, 20, 0, 0, "mixed"), ("f32", 1300, 2100, 500, 4, 24, 0, 0, "mixed"),
    ("bf16", 2304, 1003, 1900, 4, 16, 1, 1, "mixed"), ("bf16", 1500, 1600, 1800, 12, 24, 3, 0, "runs"),  # (copied: rows and W, rows)
    ("bf16", 700, 1111, 333, 9, 16, 1, 0, "runs"), ("f32", 700, 1111, 333, 9, 7, 1, 0, "mixed"), ("bf16", 190, 2048, 1032, 3, 64, 0, 0, "mixed"),
]


@pytest.mark.parametrize("case", MANY, ids=lambda s: "-".join(map(str, s)))
def test_forward_of_many_rows(ctx, case):
    t, rows, width, outs, n, r, pad, shift, order = case
    v = inputs(rows, width, outs, n, r, t, rows + width, pad, shift, order=order)
    near(forward(ctx, *v[:7], pad=pad, shift=shift), *adapter_forward(*v[:7]), width, width + r, t == "bf16")


@pytest.mark.parametrize("case", MANY, ids=lambda s: "-".join(map(str, s)))
def test_backward_of_many_rows(ctx, case):
    t, rows, width, outs, n, r, pad, shift, order = case
    v = inputs(rows, outs, width, n, r, t, rows + outs, pad, shift, order=order)
    got, want = backward(ctx, *v, pad=pad, shift=shift), adapter_backward(*v)
    near(got["dx"], *want["dx"], width, width + r, t == "bf16")
    near(got["da"], *want["da"], 0, width + rows, False)
    near(got["db"], *want["db"], 0, outs + rows, False)


APART = [("bf16", 20, 256, 136, 3, 8), ("f32", 20, 129, 63, 3, 5), ("bf16", 100, 512, 264, 4, 16), ("bf16", 100, 511, 263, 4, 24), ("f32", 100, 300, 200, 3, 24),
         ("bf16", 1500, 136, 2056, 6, 40), ("bf16", 2200, 75, 1801, 3, 8), ("bf16", 2304, 1003, 1900, 4, 16), ("f32", 2200, 72, 1800, 5, 12), ("bf16", 4001, 72, 3528, 4, 16)]


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("case", APART, ids=lambda s: "-".join(map(str, s)))
def test_an_adapter_that_is_not_finite_meets_its_own_rows_only(ctx, case, bad):
    """One element of B (which y meets) and of A (which dx meets): the other adapters' rows and gradients keep their bits."""
    t, rows, ci, co, n, r = case
    v = list(inputs(rows, ci, co, n, r, t, 7, ranks=False))
    v[2] = torch.randint(-1, n, (rows,), generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    other = v[2] != 1
    y, want = forward(ctx, *v[:7]), adapter_forward(*v[:7])
    v[4] = v[4].clone()
    v[4][1, co // 2, r // 2] = bad
    z = forward(ctx, *v[:7])
    assert torch.equal(y[other], z[other])
    assert not bool(torch.isfinite(z[~other][:, co // 2]).any())
    keep = torch.arange(co) != co // 2  # (its own rows' other sums: made in another order)
    near(z[:, keep.cuda()], *[u[:, keep] for u in want], ci, ci + r, t == "bf16")

    v = list(inputs(rows, co, ci, n, r, t, 8, ranks=False))  # (dx as wide as y was)
    v[2] = torch.where(other, v[2].clamp(max=0), 1).to(torch.int32)
    g = backward(ctx, *v)
    v[3] = v[3].clone()
    v[3][1, r // 2, co // 2] = bad
    f = backward(ctx, *v)
    assert torch.equal(g["dx"][other], f["dx"][other])
    assert not bool(torch.isfinite(f["dx"][~other][:, co // 2]).any())
    assert torch.equal(g["da"], f["da"])
    assert torch.equal(g["db"][[i for i in range(n) if i != 1]], f["db"][[i for i in range(n) if i != 1]])


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("case", APART, ids=lambda s: "-".join(map(str, s)))
def test_a_row_that_is_not_finite_meets_no_other(ctx, case, bad):
    t, rows, ci, co, n, r = case
    v = list(inputs(rows, ci, co, n, r, t, 9, ranks=False))
    at = rows // 3
    v[2][at] = 1
    v[2][at + 1] = 0
    other = torch.arange(rows, device="cuda") != at
    y, g = forward(ctx, *v[:7]), backward(ctx, *v)
    v[0], v[7] = v[0].clone(), v[7].clone()
    v[0][at, ci // 2] = bad
    v[7][at, co // 2] = bad
    z, f = forward(ctx, *v[:7]), backward(ctx, *v)
    assert torch.equal(y[other], z[other]) and not bool(torch.isfinite(z[at]).any())
    assert torch.equal(g["dx"][other], f["dx"][other]) and not bool(torch.isfinite(f["dx"][at]).any())
    rest = [i for i in range(n) if i != 1]
    assert torch.equal(g["da"][rest], f["da"][rest]) and torch.equal(g["db"][rest], f["db"][rest])
