"""wcc_distill_forward and wcc_distill_backward against the definition in 64 bits and against differences (needs an MI355X).

The log of a row's sum is off by less than (512 + 16) 2^-24 = 3.2e-5 (at most 512 terms a thread, a tree of a dozen levels, an ulp
each).  A pair's term q (log q - log p) inherits that times 1 + the magnitudes of the logarithms; a gradient's p and q are off by that
relative to themselves (their exponents' size included: below 100 here, an ulp each), and a bf16 result by half an ulp, 2^-8."""
import math

import pytest
import torch

from paper_2205_12268_amd import wcc
from tests.head_util import TYPES, around, distill, logits_like, rows_of

pytestmark = pytest.mark.gpu
TOL = 3.2e-5


@pytest.fixture(scope="module")
def ctx():
    c = wcc.Context(0)
    yield c
    c.close()


def teacher(rows, V, K, seed, holes=False, t="f32"):
    gen = torch.Generator().manual_seed(seed)
    idx = torch.stack([torch.randperm(V, generator=gen)[:K] if V < 20000 else torch.randint(0, V, (K,), generator=gen)
                       for _ in range(rows)]).to(torch.int32) if K <= V else torch.randint(0, V, (rows, K), generator=gen, dtype=torch.int32)
    z = (4 + 2 * torch.randn((rows, K), generator=gen)).to(TYPES[t])
    if holes:
        idx[torch.rand((rows, K), generator=gen) < 0.3] = -1
        z[torch.rand((rows, K), generator=gen) < 0.2] = -math.inf
        idx[0] = -1
        if K > 2:
            idx[-1, 1] = V  # outside: none
            idx[-1, 2] = idx[-1, 0]  # twice the same
    return idx.cuda(), z.cuda()


def run(ctx, x, idx, z, tau, weight=None, mode="step", pad=0, shift=0, in_place=False):
    rows, V = x.shape
    dt = wcc.BF16 if x.dtype == torch.bfloat16 else wcc.F32
    tt = wcc.BF16 if z.dtype == torch.bfloat16 else wcc.F32
    grad = x if in_place else rows_of(torch.full((rows, V), 9.0), x.dtype, pad, shift)
    d = wcc.make_distill_desc(rows, V, idx.shape[1], dt, tt, tau, ld=x.stride(0) if rows > 1 else V,
                              ld_grad=grad.stride(0) if rows > 1 else V)
    ctx.ensure_workspace(d)
    loss, stats = torch.full((rows,), 7.0, device="cuda"), torch.full((rows, 2), 7.0, device="cuda")
    if mode == "step":
        ctx.wcc_distill_forward(d, x, idx, z, loss, stats, weight, grad)
    else:
        ctx.wcc_distill_forward(d, x, idx, z, loss, stats)
        if mode == "two":
            ctx.wcc_distill_backward(d, x, idx, z, stats, weight, grad)
    torch.cuda.synchronize()
    if mode != "loss" and not in_place:
        assert bool(torch.isnan(around(grad)).all())  # nothing outside the rows was touched
    return loss.cpu().double(), stats.cpu().double(), grad


def check(ctx, x, idx, z, tau, weight=None, **kw):
    loss, stats, grad, size = distill(x, idx, z, tau, None if weight is None else weight.cpu())
    for mode in ("step", "two", "loss"):
        got_loss, got_stats, got = run(ctx, x, idx, z, tau, weight, mode, **kw)
        assert torch.equal(got_stats == -math.inf, stats == -math.inf)
        ok = stats > -math.inf
        assert bool(((got_stats - stats)[ok].abs() <= TOL * (1 + stats[ok].abs())).all())
        fine = torch.isfinite(loss)
        assert torch.equal(got_loss[~fine], loss[~fine])
        assert bool(((got_loss - loss)[fine].abs() <= TOL * size[fine]).all()), float((got_loss - loss)[fine].abs().max())
        if mode == "loss":
            continue
        w = torch.ones(len(loss)).double() if weight is None else weight.cpu().double()
        # p <= |g| + q and q <= |g| + p: where pairs are, both have their own errors
        q_mass = torch.zeros_like(grad)
        for t in range(len(loss)):
            zs = z[t].double().cpu() / tau
            keep = (idx[t].cpu() >= 0) & (idx[t].cpu() < x.shape[1]) & (zs > -math.inf)
            if bool(keep.any()):
                q_mass[t].index_add_(0, idx[t].cpu().long()[keep], torch.softmax(zs[keep], 0))
        scale = (tau * w.abs())[:, None]
        tol = 2 * TOL * (grad.abs() + 2 * scale * q_mass) + 1e-30
        if x.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * 1.001 * grad.abs()
        off = (got.double().cpu() - grad).abs()
        assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("t,tt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,V,K,tau,pad,shift", [
    (1, 1, 1, 1.0, 0, 0), (3, 2, 2, 2.0, 1, 1), (2, 9, 4, 0.5, 0, 3), (5, 64, 64, 1.0, 0, 0), (4, 1000, 17, 1.5, 5, 1),
    (3, 5003, 256, 2.0, 3, 0), (2, 30011, 100, 4.0, 0, 1), (1, 70000, 32, 1.0, 0, 0), (2, 140001, 5, 2.0, 7, 3), (130, 333, 8, 1.0, 0, 0)])
def test_sizes(ctx, t, tt, rows, V, K, tau, pad, shift):
    x = rows_of(logits_like(rows, V, rows + V), TYPES[t], pad, shift)
    idx, z = teacher(rows, V, K, V + K, t=tt)
    weight = torch.rand(rows, generator=torch.Generator().manual_seed(V)).cuda()
    check(ctx, x, idx, z, tau, weight, pad=pad, shift=shift)
    check(ctx, x, idx, z, tau)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 600, 40001, 150000])
def test_masks_and_holes(ctx, t, V):
    """Pairs that are none, indices given twice, rows without a teacher, masked logits (the loss is +inf where a pair sits on one),
    rows that a mask leaves empty, masks of the type's lowest value."""
    z = logits_like(6, V, V, masked=0.4, empty=(2,))
    z[3] = torch.finfo(TYPES[t]).min
    x = rows_of(z, TYPES[t], pad=3)
    idx, tz = teacher(6, V, 5, V, holes=True)
    weight = torch.tensor([1.0, 0.5, 2.0, 1.0, 0.0, 3.0]).cuda()
    idx[3] = -1  # (a difference of 3e38 has no finite loss)
    idx[3, 0] = 1
    check(ctx, x, idx, tz, 2.0, weight, pad=3)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(3, 1000), (1, 100001), (4, 200001)])
def test_in_place(ctx, t, rows, V):
    base = rows_of(logits_like(rows, V, 4), TYPES[t], pad=2)
    idx, z = teacher(rows, V, 16, 9)
    loss, _, grad = run(ctx, base, idx, z, 1.5, pad=2)
    for mode in ("step", "two"):
        x = rows_of(base.cpu().float(), TYPES[t], pad=2)
        loss2, _, grad2 = run(ctx, x, idx, z, 1.5, mode=mode, in_place=True)
        assert torch.equal(loss, loss2)
        if mode == "step":
            assert torch.equal(grad, grad2)
        else:
            assert float((grad.float() - grad2.float()).abs().max()) <= 2.0 ** -8 * float(grad.float().abs().max())


def test_gradient_against_differences(ctx):
    """The gradient of sum_t weight loss against central differences of the 64-bit loss: off by the third derivative, below
    weight tau^2 h^2 / tau^3 = 1e-8 at h = 1e-4, and by the gradient's own 2e-5."""
    rows, V, K, tau = 3, 37, 6, 1.7
    x = rows_of(logits_like(rows, V, 8), torch.float32)
    idx, z = teacher(rows, V, K, 3, holes=True)
    weight = torch.tensor([0.7, 1.3, 2.0]).cuda()
    _, _, grad = run(ctx, x, idx, z, tau, weight)
    base = x.double().cpu()
    for t in range(rows):
        for v in range(V):
            up, down = base.clone(), base.clone()
            up[t, v] += 1e-4
            down[t, v] -= 1e-4
            diff = (distill(up, idx, z, tau)[0][t] - distill(down, idx, z, tau)[0][t]) / 2e-4 * float(weight[t])
            assert abs(float(grad[t, v]) - float(diff)) <= 2e-5 * (abs(float(diff)) + float(weight[t]))


def test_rows_beyond_32_bit_offsets(ctx):
    V, ld, rows = 901, (1 << 30) + 3, 5
    buf = torch.empty(ld * (rows - 1) + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, V), (ld, 1))
    x.copy_(logits_like(rows, V, 11))
    idx, z = teacher(rows, V, 12, 1)
    small = rows_of(x.cpu().float(), torch.bfloat16)
    want = run(ctx, small, idx, z, 1.0)
    d = wcc.make_distill_desc(rows, V, 12, wcc.BF16, wcc.F32, 1.0, ld=ld, ld_grad=ld)
    ctx.ensure_workspace(d)
    loss = torch.zeros(rows, device="cuda")
    ctx.wcc_distill_forward(d, x, idx, z, loss, None, None, x)
    assert torch.equal(loss.cpu().double(), want[0])
    assert torch.equal(x.contiguous(), want[2].contiguous())


@pytest.mark.parametrize("rows,V", [(2, 200001), (50, 3001)])
def test_in_a_graph(ctx, rows, V):
    x = rows_of(logits_like(rows, V, 2), torch.bfloat16)
    idx, z = teacher(rows, V, 20, 2)
    d = wcc.make_distill_desc(rows, V, 20, wcc.BF16)
    own = wcc.Context(0)
    own.ensure_workspace(d)
    loss, stats, grad = torch.zeros(rows, device="cuda"), torch.zeros((rows, 2), device="cuda"), torch.zeros_like(x.contiguous())
    own.wcc_distill_forward(d, x, idx, z, loss, stats, None, grad)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        own.wcc_distill_forward(d, x, idx, z, loss, stats, None, grad)
    for seed in (3, 4, 5):
        x.copy_(logits_like(rows, V, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (loss, stats, grad)]
        own.wcc_distill_forward(d, x, idx, z, loss, stats, None, grad)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, stats, grad)))
    own.close()


def test_refusals(ctx):
    import ctypes as C
    x, z = torch.zeros((4, 100), device="cuda"), torch.zeros((4, 5), device="cuda")
    idx, loss = torch.zeros((4, 5), dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    L, h = wcc.lib(), ctx._h
    good = dict(rows=4, V=100, K=5, dtype=wcc.F32)
    ctx.ensure_workspace(wcc.make_distill_desc(**good))

    def status(args, desc):
        p = [None if v is None else C.c_void_p(v if isinstance(v, int) else v.data_ptr()) for v in args]
        return L.wcc_distill_forward(h, C.byref(desc), *p, None)

    d = wcc.make_distill_desc(**good)
    for hole in range(4):
        args = [x, idx, z, loss, None, None, None]
        args[hole] = None
        assert status(args, d) == 1
    assert status([x.data_ptr() + 1, idx, z, loss, None, None, None], d) == 8
    assert status([x, idx, z, loss, None, None, x], wcc.make_distill_desc(**good, ld_grad=101)) == 2  # in place, other stride
    for bad, want in ((dict(V=0), 2), (dict(K=0), 2), (dict(ld=99), 2), (dict(ld_grad=99), 2), (dict(dtype=wcc.I4), 3), (dict(t_dtype=9), 3),
                      (dict(temperature=0.0), 2), (dict(temperature=math.nan), 2), (dict(temperature=math.inf), 2), (dict(temperature=-1.0), 2),
                      (dict(K=257), 6), (dict(rows=-1), 2)):
        kw = dict(good)
        kw.update(bad)
        assert status([x, idx, z, loss, None, None, None], wcc.make_distill_desc(**kw)) == want, bad
    assert L.wcc_distill_backward(h, C.byref(d), x.data_ptr(), idx.data_ptr(), z.data_ptr(), None, None, x.data_ptr(), None) == 1
    ctx.wcc_distill_forward(wcc.make_distill_desc(0, 100, 5, wcc.F32), x[:0], idx[:0], z[:0], loss[:0])
    torch.cuda.synchronize()
