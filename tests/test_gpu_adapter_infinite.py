"""Infinities where the definition gives infinities: lines and operands that the kernels split into bf16 parts must not turn them into
NaN by products with parts that are 0 (needs an MI355X).  Finite results: tolerances as in test_gpu_adapter.py."""
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


SIZES = [("bf16", 20, 256, 136, 3, 8), ("f32", 20, 129, 63, 3, 5), ("bf16", 100, 512, 264, 4, 16), ("bf16", 100, 511, 263, 4, 24), ("f32", 100, 300, 200, 3, 24),
         ("bf16", 1500, 136, 2056, 6, 40), ("bf16", 2304, 1003, 1900, 4, 16), ("bf16", 4001, 72, 3528, 4, 40)]


def chosen(rows, ci, co, n, r, t, seed):
    """Adapters that pick elements of x and dy: every line is a bf16 number, its lower parts are 0."""
    v = list(inputs(rows, ci, co, n, r, t, seed, ranks=False))
    v[2] = torch.randint(-1, n, (rows,), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
    v[3], v[4] = torch.zeros_like(v[3]), torch.zeros_like(v[4])
    for j in range(r):
        v[3][:, j, j] = 1.0
        v[4][:, j, j] = 1.0
    return v


def same(got, want, n_main, n_low, narrow):
    got, (want, main, low) = got.double().cpu(), want
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    far = torch.isinf(want)
    assert torch.equal(got[far], want[far])
    fine = torch.isfinite(want) & torch.isfinite(main) & torch.isfinite(low)
    near(got[fine], want[fine], main[fine], low[fine], n_main, n_low, narrow)


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_an_adapter(ctx, size, bad):
    t, rows, ci, co, n, r = size
    v = chosen(rows, ci, co, n, r, t, 11)
    v[4][1, co // 2, r // 2] = bad
    want = adapter_forward(*v[:7])
    assert bool(torch.isinf(want[0]).any())
    same(forward(ctx, *v[:7]), want, ci, ci + r, t == "bf16")
    v = chosen(rows, co, ci, n, r, t, 12)  # (dx as wide as y was)
    v[3][1, r // 2, co // 2] = bad
    want = adapter_backward(*v)
    assert bool(torch.isinf(want["dx"][0]).any())
    same(backward(ctx, *v)["dx"], want["dx"], ci, ci + r, t == "bf16")


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_rows(ctx, size, bad):
    """x, then dy, of one row: dA and dB have infinities in one column, of the sign of the other factor."""
    t, rows, ci, co, n, r = size
    for which, name in ((0, "da"), (7, "db")):
        v = chosen(rows, ci, co, n, r, t, 13)
        at = rows // 3
        v[2][at] = 1
        v[which] = v[which].clone()
        v[which][at, v[which].shape[1] - 1] = bad
        want = adapter_backward(*v)
        assert bool(torch.isinf(want[name][0]).any())
        got = backward(ctx, *v)
        same(got["da"], want["da"], 0, co + rows, False)
        same(got["db"], want["db"], 0, ci + rows, False)


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_lines(ctx, size, bad):
    """One line of an infinite row is infinite (no element of A is 0): so are y and dB wherever B and dy are not 0."""
    t, rows, ci, co, n, _ = size
    v = list(inputs(rows, ci, co, n, 1, t, 14, ranks=False))
    at = rows // 3
    v[2][at] = 1
    v[0] = v[0].clone()
    v[0][at, ci // 2] = bad
    v[1] = torch.where(v[1] == 0, 1.0, v[1].float().abs()).to(v[1].dtype) * (1 if float(v[3][1, 0, ci // 2]) > 0 else -1)  # W x of the sign of A x
    v[4] = torch.where(v[4] == 0, 1.0, v[4].float().abs()).to(v[4].dtype)  # and B h
    want = adapter_forward(*v[:7])
    assert bool(torch.isinf(want[0][at]).all())
    same(forward(ctx, *v[:7]), want, ci, ci + 1, t == "bf16")
    want = adapter_backward(*v)
    assert bool(torch.isinf(want["db"][0][1]).any())
    same(backward(ctx, *v)["db"], want["db"], 0, ci + rows, False)


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_lines_beside_an_infinite_adapter(ctx, size, bad):
    """Infinite lines of an adapter that holds an infinity itself: outputs whose elements of B are finite have an infinity, not NaN."""
    t, rows, ci, co, n, _ = size
    v = list(inputs(rows, ci, co, n, 1, t, 15, ranks=False))
    at = rows // 3
    v[2][at] = 1
    v[0] = v[0].clone()
    v[0][at, ci // 2] = bad
    v[1] = torch.where(v[1] == 0, 1.0, v[1].float().abs()).to(v[1].dtype) * (1 if float(v[3][1, 0, ci // 2]) > 0 else -1)  # W x of the sign of A x
    v[4] = torch.where(v[4] == 0, 1.0, v[4].float().abs()).to(v[4].dtype)  # and B h
    v[4][1, co // 2, 0] = math.inf
    want = adapter_forward(*v[:7])
    assert bool(torch.isinf(want[0][at]).all())
    same(forward(ctx, *v[:7]), want, ci, ci + 1, t == "bf16")
