"""wcc_token_scores against its definition in 64 bits (needs an MI355X).

Indices have to be equal.  A log probability's error: its sum has at most 512 terms a thread and a tree of a dozen levels, each
addition and each exponential with an ulp at most, so log S is off by less than (512 + 16) 2^-24 = 3.2e-5; differences and
logarithms add ulps of the value itself.  Hence 3.2e-5 (1 + |value|)."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, logits_like, rows_of, scores

pytestmark = pytest.mark.gpu
TOL = 3.2e-5


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def call(ctx, x, tokens, top):
    rows, V = x.shape
    ld = x.stride(0) if rows > 1 else V
    d = wcc.make_scores_desc(rows, V, top, wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32, ld=ld)
    ctx.ensure_workspace(d)
    out = [torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda"),
           torch.full((rows, top), -7, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda")]
    ctx.wcc_token_scores(d, x, tokens, *out)
    torch.cuda.synchronize()
    return [o.cpu() for o in out]


def near(got, want):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got == -math.inf, want == -math.inf)
    fine = torch.isfinite(want)
    assert bool(((got - want).abs()[fine] <= TOL * (1 + want[fine].abs())).all()), float((got - want).abs()[fine].max())


def check(ctx, x, tokens, top):
    lp, ent, idx, tlp = call(ctx, x, tokens, top)
    wlp, went, widx, wtlp = scores(x, tokens, top)
    near(lp, wlp)
    near(ent, went)
    assert torch.equal(idx.long(), widx)
    near(tlp, wtlp)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top,pad,shift", [
    (1, 1, 1, 0, 0), (3, 2, 2, 1, 1), (2, 7, 7, 0, 3), (5, 63, 5, 3, 0), (4, 64, 64, 0, 0), (3, 65, 20, 0, 1), (1, 1000, 0, 0, 0),
    (2, 4099, 50, 5, 2), (1, 8192, 64, 0, 0), (7, 30011, 8, 1, 1), (1, 131072, 20, 0, 0), (2, 150001, 64, 8, 5), (300, 257, 3, 0, 0)])
def test_sizes(ctx, t, rows, V, top, pad, shift):
    x = rows_of(logits_like(rows, V, 100 * rows + V), TYPES[t], pad, shift)
    tokens = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(V), dtype=torch.int32).cuda()
    check(ctx, x, tokens, top)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 300, 9001, 140000])
def test_masks(ctx, t, V):
    z = logits_like(6, V, V, masked=0.5, empty=(2,))
    z[3] = torch.finfo(TYPES[t]).min      # a mask of the type's lowest value everywhere: still a distribution
    z[4, 1:] = torch.finfo(TYPES[t]).min  # and everywhere but at one place
    z[5, :] = -math.inf
    z[5, V - 1] = 3.0
    x = rows_of(z, TYPES[t])
    tokens = torch.tensor([0, V - 1, 1, 2, 0, V - 1], dtype=torch.int32).cuda()
    check(ctx, x, tokens, min(V, 9))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 513, 70000])
def test_ties_go_to_the_lower_index(ctx, t, V):
    z = torch.zeros((5, V))
    z[1] = (torch.arange(V) % 3).float()
    z[2] = torch.arange(V).float()          # rising
    z[3] = -(torch.arange(V) // 5).float()  # falling in steps
    z[4, ::2] = -0.0                        # equal to the zeros between them
    x = rows_of(z, TYPES[t], pad=1)
    check(ctx, x, torch.zeros(5, dtype=torch.int32).cuda(), min(V, 33))


def test_large_values_and_none(ctx):
    z = logits_like(6, 500, 5)
    z[0] *= 1e30
    z[1, 7] = math.inf
    z[2, 9] = math.nan
    z[3] -= 1e4
    z[4, 100] = 3e38
    x = rows_of(z, torch.float32)
    tokens = torch.tensor([3, 3, 3, -1, 500, 499], dtype=torch.int32).cuda()
    check(ctx, x, tokens, 4)


def test_only_what_is_asked_for(ctx):
    x = rows_of(logits_like(4, 1001, 1), torch.float32)
    d = wcc.make_scores_desc(4, 1001, 0, wcc.F32)
    ctx.ensure_workspace(d)
    ent = torch.zeros(4, device="cuda")
    ctx.wcc_token_scores(d, x, None, None, ent)
    near(ent.cpu(), scores(x, torch.zeros(4), 0)[1])
    d = wcc.make_scores_desc(4, 1001, 3, wcc.F32)
    ctx.ensure_workspace(d)
    idx = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    ctx.wcc_token_scores(d, x, None, None, None, idx)
    assert torch.equal(idx.cpu().long(), scores(x, torch.zeros(4), 3)[2])
    ctx.wcc_token_scores(wcc.make_scores_desc(0, 1001, 3, wcc.F32), x[:0], None, None, None, idx[:0])


def test_equal_calls_give_equal_bits(ctx):
    x = rows_of(logits_like(9, 50001, 3), torch.bfloat16)
    tokens = torch.arange(9, dtype=torch.int32).cuda()
    first = call(ctx, x, tokens, 16)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, call(ctx, x, tokens, 16)))


def test_rows_beyond_32_bit_offsets(ctx):
    """Rows so far apart that the last one begins 2^32 elements into its buffer and beyond."""
    V, ld, rows = 777, (1 << 30) + 5, 5
    buf = torch.empty(ld * (rows - 1) + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, V), (ld, 1))
    x.copy_(logits_like(rows, V, 11))
    d = wcc.make_scores_desc(rows, V, 6, wcc.BF16, ld=ld)
    ctx.ensure_workspace(d)
    tokens = torch.arange(rows, dtype=torch.int32).cuda()
    lp, ent = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    idx, tlp = torch.zeros((rows, 6), dtype=torch.int32, device="cuda"), torch.zeros((rows, 6), device="cuda")
    ctx.wcc_token_scores(d, x, tokens, lp, ent, idx, tlp)
    want = scores(x.contiguous(), tokens, 6)
    near(lp.cpu(), want[0])
    near(ent.cpu(), want[1])
    assert torch.equal(idx.cpu().long(), want[2])


@pytest.mark.parametrize("rows,V", [(2, 100000), (64, 5000)])
def test_in_a_graph_and_on_another_stream(ctx, rows, V):
    x = rows_of(logits_like(rows, V, 2), torch.bfloat16)
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    d = wcc.make_scores_desc(rows, V, 8, wcc.BF16)
    own = wcc.Context(0)
    own.ensure_workspace(d)
    lp, ent = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    idx, tlp = torch.zeros((rows, 8), dtype=torch.int32, device="cuda"), torch.zeros((rows, 8), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        own.wcc_token_scores(d, x, tokens, lp, ent, idx, tlp)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        own.wcc_token_scores(d, x, tokens, lp, ent, idx, tlp)
    for seed in (3, 4, 5):
        x.copy_(logits_like(rows, V, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (lp, ent, idx, tlp)]
        own.wcc_token_scores(d, x, tokens, lp, ent, idx, tlp)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (lp, ent, idx, tlp)))
        assert torch.equal(idx.cpu().long(), scores(x, tokens, 8)[2])
    own.close()


def test_refusals(ctx):
    x = torch.zeros((4, 100), device="cuda")
    out = torch.zeros(4, device="cuda")
    idx = torch.zeros((4, 5), dtype=torch.int32, device="cuda")
    L, h = wcc.lib(), ctx._h
    import ctypes as C

    def status(desc, logits, tokens, lp, ent, ti, tl):
        p = [None if v is None else C.c_void_p(v if isinstance(v, int) else v.data_ptr()) for v in (logits, tokens, lp, ent, ti, tl)]
        return L.wcc_token_scores(h, C.byref(desc), *p, None)

    good = wcc.make_scores_desc(4, 100, 5, wcc.F32)
    ctx.ensure_workspace(good)
    assert status(good, None, None, None, out, idx, None) == 1
    assert status(good, x, None, out, None, idx, None) == 1       # log probabilities of no tokens
    assert status(good, x, None, None, out, None, None) == 1      # no room for the alternatives
    assert status(good, x.data_ptr() + 2, None, None, out, idx, None) == 8
    for bad, want in ((dict(V=0), 2), (dict(ld=99), 2), (dict(top=101, V=100), 2), (dict(top=-1), 2), (dict(dtype=wcc.I8), 3),
                      (dict(rows=-1), 2), (dict(top=65), 6)):
        kw = dict(rows=4, V=100, top=5, dtype=wcc.F32)
        kw.update(bad)
        assert status(wcc.make_scores_desc(**kw), x, None, None, out, idx, None) == want, bad
    fresh = wcc.Context(0)
    big = wcc.make_scores_desc(1, 131072, 5, wcc.F32)
    if wcc.scores_workspace_bytes(big):
        y = torch.zeros((1, 131072), device="cuda")
        with pytest.raises(wcc.WccError):
            fresh.wcc_token_scores(big, y, None, None, out[:1], idx[:1])
    fresh.close()
    torch.cuda.synchronize()
