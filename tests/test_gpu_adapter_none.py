"""wcc_adapter_forward and wcc_adapter_backward without adapters, their A and B NULL: the projection alone, on every route (needs an
MI355X).  Tolerances as in test_gpu_adapter.py."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, adapter_backward, adapter_forward, around, rows_of
from tests.test_gpu_adapter import inputs, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("n,r", [(0, 0), (3, 16)])
@pytest.mark.parametrize("rows,ci,co,pad,shift", [(1, 64, 40, 0, 0), (20, 512, 264, 0, 0), (20, 300, 137, 3, 1), (33, 129, 63, 1, 1), (64, 1024, 520, 8, 8),
                                                  (65, 96, 160, 0, 0), (130, 75, 301, 1, 1), (1500, 264, 2056, 0, 0)])
def test_without_adapters(ctx, t, n, r, rows, ci, co, pad, shift):
    x, w, _, a, b, _, _, dy = inputs(rows, ci, co, 1, 1, t, rows + ci, pad, shift)
    none = torch.full((rows,), -1, dtype=torch.int32)
    y, dx = rows_of(torch.full((rows, co), 9.0), TYPES[t], pad, shift), rows_of(torch.full((rows, ci), 9.0), TYPES[t], pad, shift)
    da, db = torch.full((n, r, ci), 9.0, device="cuda"), torch.full((n, co, r), 9.0, device="cuda")
    d = wcc.make_adapter_desc(rows, ci, co, n, r, wcc.BF16 if t == "bf16" else wcc.F32, ldx=ci + pad, ldy=co + pad)
    ctx.ensure_workspace(d)
    ctx._ws.fill_(255)
    ctx.wcc_adapter_forward(d, x, w, None, None, None, None, None, y)
    ctx.wcc_adapter_backward(d, x, w, None, None, None, None, None, dy, dx, da if n else None, db if n else None)
    torch.cuda.synchronize()
    assert bool(torch.isnan(around(y)).all()) and bool(torch.isnan(around(dx)).all())
    near(y, *adapter_forward(x, w, none, a, b, None, None), ci, ci, t == "bf16")
    near(dx, *adapter_backward(x, w, none, a, b, None, None, dy)["dx"], co, co, t == "bf16")
    assert not bool(da.any()) and not bool(db.any())
    only = torch.full_like(dx, 9.0)
    if only.stride() == dx.stride():
        ctx.wcc_adapter_backward(d, None, w, None, None, None, None, None, dy, only)  # (no x: dx does not need it)
        assert torch.equal(only, dx)
