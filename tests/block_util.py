"""The operators of a block on rows in 64 bits, from their definitions, with bounds of what fp32 arithmetic loses beside them."""
from __future__ import annotations

import math

import torch

from paper_2205_12268_amd import wcc

U = 2.0 ** -24  # half a step of fp32
ACTS = {"none": wcc.ACT_NONE, "relu": wcc.ACT_RELU, "silu": wcc.ACT_SILU, "gelu": wcc.ACT_GELU}
NARROW = 2.0 ** -8  # half a step of bf16, relative


def act(z, name):
    """(act(z), act'(z)) in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.where(z > 0, z, 0.0), (z > 0).double()
    if name == "silu":
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        return z * p, p * (1 + z * q)
    below = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z * below, below + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


# What the kernels' value and slope are off by at an exact z: the hardware's exponential and reciprocal are off by a step each, the
# exponent's rounding by |z| / 2 steps of it (which only counts where the exponential is of the size of 1 or less beside 1), erf by
# 1.5e-7 = 2.6 U.  |d value / dz| <= 1.13, |d slope / dz| <= 0.8 (relu jumps at 0; tests of it keep away from there).
def act_error(z, ez):
    """(bound for the value, bound for the slope) at z known to ez."""
    return 1.13 * ez + 12 * U * (1 + z.abs()), 0.8 * ez + 16 * U * (1 + z.abs())


# ---- rows in 8 bits ------------------------------------------------------------------------------------
def kept(x):
    """(codes, steps, values in 64 bits) of rows, block by block as the definition says."""
    x = x.double().cpu()
    rows, width = x.shape
    room = wcc.kept_room(width)
    v = torch.zeros((rows, room), dtype=torch.float64)
    v[:, :width] = x
    codes, steps = torch.zeros((rows, room), dtype=torch.int8), torch.zeros((rows, room // 32), dtype=torch.uint8)
    values = torch.zeros_like(v)
    for t in range(rows):
        for b in range(room // 32):
            part = v[t, 32 * b:32 * b + 32]
            if not bool(torch.isfinite(part).all()):
                steps[t, b] = 255
                values[t, 32 * b:32 * b + 32] = math.nan
                continue
            top = float(part.abs().max())
            e = max(math.frexp(top)[1] - 7, -126) if top > 0 else -126
            if top / 2.0 ** e >= 127.5 and e < 121:
                e += 1
            q = (part / 2.0 ** e).round().clamp(-127, 127)
            codes[t, 32 * b:32 * b + 32] = q.to(torch.int8)
            steps[t, b] = e + 127
            values[t, 32 * b:32 * b + 32] = q * 2.0 ** e
    return codes, steps, values[:, :width]


def kept_on_gpu(x):
    codes, steps, values = kept(x)
    return codes.cuda(), steps.cuda(), values


# ---- group norm ----------------------------------------------------------------------------------------
def group_norm(x, samples, groups, gamma, beta, counts, eps, name, dy=None, kept_x=None):
    """{name: (result, bound of fp32's loss)}: y, mean, rstd, and with dy the gradients, from kept_x if it is given.  Rows that are not
    there are NaN in y and dx."""
    x = x.double().cpu()
    rows, C = x.shape
    pixels, per = rows // samples, C // groups
    g = torch.ones(C).double() if gamma is None else gamma.double().cpu()
    b = torch.zeros(C).double() if beta is None else beta.double().cpu()
    eps = float(torch.tensor(eps, dtype=torch.float32))
    out = {k: [torch.full_like(x, math.nan), torch.full_like(x, math.nan)] for k in ("y", "dx")}
    stats = torch.zeros((samples, groups, 2)).double()
    dgamma, dbeta, egamma, ebeta = (torch.zeros(C).double() for _ in range(4))
    for i in range(samples):
        n = pixels if counts is None else min(max(int(counts[i]), 0), pixels)
        stats[i, :, 1] = 1 / math.sqrt(eps)
        if n == 0:
            continue
        at = slice(i * pixels, i * pixels + n)
        wide = lambda v: v.repeat_interleave(per)[None]  # noqa: E731  (a group's value for each of its channels)
        mean_of = lambda v: wide(v.reshape(n, groups, per).mean(dim=(0, 2)))  # noqa: E731
        v = x[at]
        mean = v.reshape(n, groups, per).mean(dim=(0, 2))
        var = ((v - wide(mean)) ** 2).reshape(n, groups, per).mean(dim=(0, 2))
        rstd = 1 / (var + eps).sqrt()
        stats[i, :, 0], stats[i, :, 1] = mean, rstd

        def normed(v):
            """xh, z and what fp32 loses of them: the rounding of mean, of the difference, of rstd (2), of products and sum"""
            xh = (v - wide(mean)) * wide(rstd)
            exh = U * (wide(rstd) * wide(mean).abs() + 6 * xh.abs())
            z = xh * g + b
            return xh, exh, z, g.abs() * exh + 4 * U * ((xh * g).abs() + b.abs())
        xh, exh, z, ez = normed(v)
        value, _ = act(z, name)
        out["y"][0][at], out["y"][1][at] = value, act_error(z, ez)[0]
        if dy is None:
            continue
        if kept_x is not None:
            xh, exh, z, ez = normed(kept_x.double().cpu()[at])
        top = dy.double().cpu()[at]
        dz = top * act(z, name)[1]
        edz = top.abs() * act_error(z, ez)[1] + U * dz.abs()
        d, ed = dz * g, edz * g.abs() + U * (dz * g).abs()
        m1, m2 = mean_of(d), mean_of(d * xh)
        # (sums: fp32 over four, then fp64)
        em1 = mean_of(ed + 4 * U * d.abs())
        em2 = mean_of(ed * xh.abs() + d.abs() * exh + 5 * U * (d * xh).abs())
        r = wide(rstd)
        out["dx"][0][at] = r * (d - m1 - xh * m2)
        out["dx"][1][at] = r * (ed + em1 + xh.abs() * em2 + exh * m2.abs() + 8 * U * (d.abs() + m1.abs() + (xh * m2).abs()))
        dgamma += (dz * xh).sum(dim=0)
        dbeta += dz.sum(dim=0)
        egamma += (edz * xh.abs() + dz.abs() * exh + 5 * U * (dz * xh).abs()).sum(dim=0)
        ebeta += (edz + 4 * U * dz.abs()).sum(dim=0)
    res = {"y": out["y"], "stats": (stats, 2 * U * stats.abs() + 1e-30)}
    if dy is not None:
        res |= {"dx": out["dx"], "dgamma": (dgamma, egamma + U * dgamma.abs()), "dbeta": (dbeta, ebeta + U * dbeta.abs())}
    return res


# ---- the gated block -----------------------------------------------------------------------------------
def projected(x, w):
    """w x and a bound of what fp32 sums in any order, joined from up to 64 ranges, lose of it."""
    x, w = x.double().cpu(), w.double().cpu()
    return x @ w.t(), (x.shape[1] + 64) * U * (x.abs() @ w.abs().t())


def gated_forward(x, w_gate, w_up, name):
    """{"y", "g", "u"}: (result, bound)."""
    g, eg = projected(x, w_gate)
    u, eu = projected(x, w_up)
    value, _ = act(g, name)
    ev, _ = act_error(g, eg)
    return {"y": (value * u, ev * (u.abs() + eu) + value.abs() * eu + U * (value * u).abs()), "g": (g, eg), "u": (u, eu)}


def gated_backward(x, w_gate, w_up, name, dy, narrow, kept_gu=None):
    """{"dx", "dw_gate", "dw_up"}: (result, bound); narrow: dg and du are rounded to bf16, twice (16 bits) where they are fewer than 2^17
    values each; kept_gu: values of g and u."""
    (g, eg), (u, eu) = (projected(x, w) for w in (w_gate, w_up)) if kept_gu is None else ((v.double().cpu(), 0 * v.double().cpu()) for v in kept_gu)
    x, dy, wg, wu = (v.double().cpu() for v in (x, dy, w_gate, w_up))
    value, slope = act(g, name)
    ev, es = act_error(g, eg)
    dg, du = dy * u * slope, dy * value
    edg = dy.abs() * (eu * (slope.abs() + es) + u.abs() * es) + 2 * U * dg.abs()
    edu = dy.abs() * ev + U * du.abs()
    rows, n = dy.shape
    if narrow:
        off = 1.001 * (NARROW ** 2 if rows * n < 1 << 17 else NARROW)
        edg, edu = edg + off * (dg.abs() + edg), edu + off * (du.abs() + edu)
    sums = lambda k, mag: (k + 64) * U * mag * 1.01  # noqa: E731
    return {"dx": (dg @ wg + du @ wu, edg @ wg.abs() + edu @ wu.abs() + sums(4 * n, dg.abs() @ wg.abs() + du.abs() @ wu.abs())),
            "dw_gate": (dg.t() @ x, edg.t() @ x.abs() + sums(2 * rows, dg.abs().t() @ x.abs())),
            "dw_up": (du.t() @ x, edu.t() @ x.abs() + sums(2 * rows, du.abs().t() @ x.abs()))}


def near(got, want, narrow, what=""):
    """got within the bound of want, and with `narrow` half a step of bf16 beside it."""
    value, tol = want
    tol = tol + 1e-37
    if narrow:
        tol = tol + NARROW * 1.001 * (value.abs() + tol)
    off = (got.double().cpu() - value).abs()
    assert bool((off <= tol).all()), (what, float((off / tol).nan_to_num(math.inf).max()))
