"""The operators of a block on rows, host side: argument checks and workspaces, which need no GPU."""
import ctypes as C

import pytest

from paper_2205_12268_amd import wcc

NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED, ALIGN = 1, 2, 3, 5, 6, 8


@pytest.mark.parametrize("kw,status", [
    (dict(samples=-1), SHAPE), (dict(pixels=0), SHAPE), (dict(Cc=0), SHAPE), (dict(Cc=(1 << 20) + 1), SHAPE), (dict(groups=0), SHAPE),
    (dict(groups=5), SHAPE), (dict(eps=0.0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(act=4), DTYPE), (dict(act=-1), DTYPE), (dict(dtype=wcc.I8), DTYPE), (dict(ldx=31), SHAPE), (dict(ldy=31), SHAPE),
    (dict(ldx=1 << 31), SHAPE), (dict(samples=1 << 16, pixels=1 << 15), SHAPE), (dict(samples=1 << 22, pixels=1, groups=4), SHAPE),
])
def test_group_norm_descriptors(kw, status):
    base = dict(samples=2, pixels=10, Cc=32, groups=4, dtype=wcc.BF16)
    out = C.c_size_t(0)
    assert wcc.lib().wcc_group_norm_workspace_bytes(C.byref(wcc.make_group_norm_desc(**(base | kw))), C.byref(out)) == status
    assert wcc.lib().wcc_group_norm_workspace_bytes(C.byref(wcc.make_group_norm_desc(**base)), C.byref(out)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(C_in=0), SHAPE), (dict(C_out=0), SHAPE), (dict(C_in=(1 << 20) + 1), SHAPE),
    (dict(ldx=15), SHAPE), (dict(ldy=23), SHAPE), (dict(act=9), DTYPE), (dict(dtype=wcc.I4), DTYPE),
    (dict(C_in=1 << 18, C_out=1 << 18), UNSUPPORTED), (dict(rows=(1 << 31) - 1, C_out=64 * 1024), UNSUPPORTED), (dict(rows=(1 << 31) - 1, C_in=64 * 1024), UNSUPPORTED),
])
def test_gated_descriptors(kw, status):
    base = dict(rows=5, C_in=16, C_out=24, dtype=wcc.F32)
    out = C.c_size_t(0)
    assert wcc.lib().wcc_gated_workspace_bytes(C.byref(wcc.make_gated_desc(**(base | kw))), C.byref(out)) == status


def calls(ctx):
    """(name, call with its arguments in a list, places of the pointers that may not be missing, places checked for 16 bytes, for 4)"""
    L, p = wcc.lib(), 4096  # (an address that nobody follows: every call below is refused)
    rows = wcc.make_rows_desc(3, 40, wcc.F32)
    norm = wcc.make_group_norm_desc(2, 10, 32, 4, wcc.F32)
    gated = wcc.make_gated_desc(300, 2048, 24, wcc.F32, train=True)
    return [
        ("wcc_rows_keep", L.wcc_rows_keep, [ctx, C.byref(rows), p, p, p, None], (2, 3, 4), (3,), (2,)),
        ("wcc_rows_restore", L.wcc_rows_restore, [ctx, C.byref(rows), p, p, p, None], (2, 3, 4), (2,), (4,)),
        ("wcc_group_norm_forward", L.wcc_group_norm_forward, [ctx, C.byref(norm), p, p, p, p, 2 * p, p, p, p, None], (2, 6, 8, 9), (8,), (2, 3, 4, 5, 6, 7)),
        ("wcc_group_norm_backward", L.wcc_group_norm_backward, [ctx, C.byref(norm), None, p, p, p, p, p, p, p, 2 * p, p, p, None], (3, 4, 8, 9), (3,),
         (5, 6, 7, 8, 9, 10, 11, 12)),
        ("wcc_gated_forward", L.wcc_gated_forward, [ctx, C.byref(gated), p, p, p, p, p, p, None], (2, 3, 4, 5, 6, 7), (6,), (2, 3, 4, 5)),
        ("wcc_gated_backward", L.wcc_gated_backward, [ctx, C.byref(gated), None, p, p, p, p, p, p, p, p, p, p, None], (3, 4, 5, 6, 8, 9), (3, 7),
         (5, 6, 9, 10, 11, 12)),
    ]


def test_refusals():
    """Missing and misaligned tensors, no descriptor, no workspace: refused before anything is enqueued (there is no GPU here)."""
    room = (C.c_char * 64)()  # (a context that is only looked at: no device, no workspace)
    ctx = C.cast(room, C.c_void_p)
    for name, call, args, needed, on_16, on_4 in calls(ctx):
        def status(at, value):
            return call(*[value if i == at else a for i, a in enumerate(args)])
        assert status(0, None) == NULL and status(1, None) == NULL, name
        for i in needed:
            assert status(i, None) == NULL, (name, i)
        for i in on_16:
            assert status(i, 4096 + 4) == ALIGN, (name, i)
        for i in on_4:
            assert status(i, 4096 + 2) == ALIGN, (name, i)
        if not name.startswith("wcc_rows"):
            assert call(*args) == WORKSPACE, name


def test_nothing_to_do():
    """No rows, and no gradient asked for."""
    room = (C.c_char * 64)()
    ctx, L, p = C.cast(room, C.c_void_p), wcc.lib(), 4096
    assert L.wcc_rows_keep(ctx, C.byref(wcc.make_rows_desc(0, 4, wcc.F32)), None, None, None, None) == 0
    assert L.wcc_rows_restore(ctx, C.byref(wcc.make_rows_desc(0, 4, wcc.F32)), None, None, None, None) == 0
    none = wcc.make_group_norm_desc(0, 5, 8, 2, wcc.F32)
    assert L.wcc_group_norm_forward(ctx, C.byref(none), *[None] * 9) == 0
    assert L.wcc_group_norm_backward(ctx, C.byref(none), *[None] * 12) == 0
    some = wcc.make_group_norm_desc(1, 5, 8, 2, wcc.F32)
    assert L.wcc_group_norm_backward(ctx, C.byref(some), p, None, None, None, None, None, p, p, None, None, None, None) == 0
    assert L.wcc_gated_forward(ctx, C.byref(wcc.make_gated_desc(0, 4, 4, wcc.F32)), *[None] * 7) == 0
    assert L.wcc_gated_backward(ctx, C.byref(wcc.make_gated_desc(3, 4, 4, wcc.F32)), p, None, None, p, p, None, None, p, None, None, None, None) == 0


def test_in_place_needs_equal_strides():
    room = (C.c_char * 64)()
    ctx, L, p = C.cast(room, C.c_void_p), wcc.lib(), 4096
    d = wcc.make_group_norm_desc(1, 5, 8, 2, wcc.F32, ldy=9)
    assert L.wcc_group_norm_forward(ctx, C.byref(d), p, None, None, None, p, None, None, None, None) == SHAPE
    assert L.wcc_group_norm_backward(ctx, C.byref(d), 2 * p, None, None, None, None, None, p, p, p, None, None, None) == SHAPE


@pytest.mark.parametrize("t", [wcc.F32, wcc.BF16])
def test_workspaces_are_whole_blocks(t):
    for rows in (0, 1, 64, 511, 5000, 1 << 19):
        for width in (1, 63, 640, 5003, 1 << 17):
            for train in (False, True):
                n = wcc.gated_workspace_bytes(wcc.make_gated_desc(rows, width, 777, t, train=train))
                assert n >= 0 and n % 256 == 0
                assert not train or n >= rows * 2 * 777 * (4 if t == wcc.F32 else 2)
            for samples in (0, 1, 7):
                n = wcc.group_norm_workspace_bytes(wcc.make_group_norm_desc(samples, max(rows, 1), width, 1, t))
                assert n % 256 == 0 and (n > 0) == (samples > 0)
