"""The binding of the operators of a block on rows, without a GPU."""
import ctypes as C

import torch

from paper_2205_12268_amd import wcc


def test_rows_need_no_workspace():
    """A program that asks for the workspace of each of its descriptors may ask for this one's."""
    ctx = wcc.Context.__new__(wcc.Context)  # (no device here)
    ctx._h, ctx.device, ctx._ws = C.c_void_p(), 0, torch.empty(16, dtype=torch.uint8)
    before = ctx._ws
    assert ctx.ensure_workspace(wcc.make_rows_desc(1000, 40, wcc.BF16)) == 0
    assert ctx._ws is before
