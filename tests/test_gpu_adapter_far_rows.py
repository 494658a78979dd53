"""The projection with adapters on rows whose last ones begin beyond 2^32 elements, on the routes of few and of many rows, both
directions (needs an MI355X and 30 GB of it).  Tolerances as in test_gpu_adapter.py."""
import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, adapter_backward, adapter_forward
from tests.test_gpu_adapter import inputs, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def apart(values, ld):
    rows, width = values.shape
    out = torch.empty(ld * (rows - 1) + width, dtype=values.dtype, device="cuda").as_strided((rows, width), (ld, 1))
    out.copy_(values)
    return out


@pytest.mark.parametrize("t,rows,odd", [("bf16", 4, 0), ("bf16", 40, 0), ("bf16", 40, 1), ("f32", 40, 0), ("bf16", 100, 0), ("bf16", 100, 1), ("f32", 130, 0)])
def test_both_directions(ctx, t, rows, odd):
    ci, co, n, r = 64, 72, 3, 8
    ld = ((1 << 32) // (rows - 1) + 77) // 8 * 8 + odd
    assert (rows - 1) * ld > 1 << 32 and ld < 1 << 31
    v = inputs(rows, ci, co, n, r, t, rows, ranks=False)
    x, dy = apart(v[0], ld), apart(v[7], ld)
    out = torch.empty(ld * (rows - 1) + co, dtype=TYPES[t], device="cuda")
    y, dx = out.as_strided((rows, co), (ld, 1)), out.as_strided((rows, ci), (ld, 1))
    da, db = torch.empty((n, r, ci), device="cuda"), torch.empty((n, co, r), device="cuda")
    d = wcc.make_adapter_desc(rows, ci, co, n, r, wcc.BF16 if t == "bf16" else wcc.F32, ldx=ld, ldy=ld)
    ctx.ensure_workspace(d)
    ctx.wcc_adapter_forward(d, x, *v[1:7], y)
    near(y, *adapter_forward(*v[:7]), ci, ci + r, t == "bf16")
    ctx.wcc_adapter_backward(d, x, *v[1:7], dy, dx, da, db)
    want = adapter_backward(*v)
    near(dx, *want["dx"], co, co + r, t == "bf16")
    near(da, *want["da"], 0, co + rows, False)
    near(db, *want["db"], 0, ci + rows, False)


def test_strides_from_2_31_on_are_refused(ctx):
    x = torch.zeros((2, 64), device="cuda")
    w, y = torch.zeros((8, 64), device="cuda"), torch.zeros((2, 8), device="cuda")
    for ldx, ldy in ((1 << 31, 8), (64, 1 << 31)):
        d = wcc.make_adapter_desc(2, 64, 8, 0, 0, wcc.F32, ldx=ldx, ldy=ldy)
        with pytest.raises(wcc.WccError) as e:
            wcc.adapter_workspace_bytes(d)
        assert e.value.status == 2
        assert wcc.lib().wcc_adapter_forward(ctx._h, d, x.data_ptr(), w.data_ptr(), None, None, None, None, None, y.data_ptr(), None) == 2
