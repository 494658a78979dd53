"""The operators of a model's head in 64 bits, row by row from their definitions, and inputs for their tests."""
from __future__ import annotations

import math

import torch

from paper_2205_12268_amd import wcc

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": wcc.F32, "bf16": wcc.BF16}


def rows_of(values, dtype, pad=0, shift=0):
    """`values` [rows, width] on the GPU in `dtype`, rows width + pad apart, the first `shift` elements into its buffer; all
    else there is NaN."""
    rows, width = values.shape
    buf = torch.full((rows * (width + pad) + shift + 8,), math.nan, dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(values)
    return view


def around(view, buf_value=math.nan):
    """All elements of a view's buffer that lie outside the view."""
    flat = torch.empty(0, dtype=view.dtype, device=view.device).set_(view.untyped_storage())
    mask = torch.ones_like(flat, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return flat[mask]


# ---- adapters ------------------------------------------------------------------------------------------
def adapter_forward(x, w, of_row, a, b, ranks, scale):
    """(y, sum of the magnitudes of W's products, the same of the adapter's), all in 64 bits on the CPU."""
    x, w, a, b = (v.double().cpu() for v in (x, w, a, b))
    y, main = x @ w.t(), x.abs() @ w.abs().t()
    low = torch.zeros_like(y)
    for t, i in enumerate(of_row.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        r = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        f = 1.0 if scale is None else float(scale[i])
        y[t] += f * (b[i, :, :r] @ (a[i, :r] @ x[t]))
        low[t] = abs(f) * (b[i, :, :r].abs() @ (a[i, :r].abs() @ x[t].abs()))
    return y, main, low


def adapter_backward(x, w, of_row, a, b, ranks, scale, dy):
    """{name: (gradient, sum of magnitudes of W's products, of the adapter's)}."""
    x, w, a, b, dy = (v.double().cpu() for v in (x, w, a, b, dy))
    dx, main, low = dy @ w, dy.abs() @ w.abs(), torch.zeros_like(x)
    da, db, ma, mb = torch.zeros_like(a), torch.zeros_like(b), torch.zeros_like(a), torch.zeros_like(b)
    for t, i in enumerate(of_row.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        r = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        f = 1.0 if scale is None else float(scale[i])
        g, gm = f * (b[i, :, :r].t() @ dy[t]), abs(f) * (b[i, :, :r].abs().t() @ dy[t].abs())
        h, hm = f * (a[i, :r] @ x[t]), abs(f) * (a[i, :r].abs() @ x[t].abs())
        dx[t] += a[i, :r].t() @ g
        low[t] = a[i, :r].abs().t() @ gm
        da[i, :r] += torch.outer(g, x[t])
        ma[i, :r] += torch.outer(gm, x[t].abs())
        db[i, :, :r] += torch.outer(dy[t], h)
        mb[i, :, :r] += torch.outer(dy[t].abs(), hm)
    return {"dx": (dx, main, low), "da": (da, torch.zeros_like(ma), ma), "db": (db, torch.zeros_like(mb), mb)}


# ---- scores --------------------------------------------------------------------------------------------
def scores(logits, tokens, top):
    """(logprob, entropy, top_idx, top_logprob) in 64 bits on the CPU."""
    x = logits.double().cpu()
    m = x.amax(dim=1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    total = (x - m).exp().sum(dim=1, keepdim=True).log()
    logp = torch.where(x == -math.inf, -math.inf, (x - m) - total)  # (m and the sum apart: m may be 3e38)
    logp[torch.isnan(total)[:, 0]] = math.nan
    p = logp.exp()
    ent = -torch.where(p == 0, 0.0, p * logp).sum(dim=1)
    given = tokens.long().cpu()
    inside = (given >= 0) & (given < x.shape[1])
    lp = torch.where(inside, logp.gather(1, given.clamp(0, x.shape[1] - 1)[:, None])[:, 0], math.nan)
    rank = torch.where(torch.isnan(x), math.inf, x)
    # NaN before +inf, larger before smaller, lower index first
    order = torch.stack([torch.tensor(sorted(range(x.shape[1]), key=lambda v, r=r: (not math.isnan(x[r, v]), -float(rank[r, v]), v))[:top],
                                      dtype=torch.int64) for r in range(x.shape[0])]) if top else torch.zeros((len(x), 0), dtype=torch.int64)
    return lp, ent, order, logp.gather(1, order)


# ---- distillation --------------------------------------------------------------------------------------
def distill(logits, t_idx, t_logit, tau, weight=None):
    """(loss, (largest, log of the sum beside it), dlogits, what a loss's error is relative to) in 64 bits on the CPU, row by row."""
    x = logits.double().cpu() / tau
    z, idx = t_logit.double().cpu() / tau, t_idx.cpu()
    rows, V = x.shape
    loss, stats, grad = torch.zeros(rows).double(), torch.zeros((rows, 2)).double(), torch.zeros_like(x)
    size = torch.zeros(rows).double()
    for t in range(rows):
        m = x[t].max()
        total = (x[t] - m).exp().sum().log() if m > -math.inf else m
        stats[t, 0], stats[t, 1] = m, total
        pairs = [(int(v), float(l)) for v, l in zip(idx[t], z[t]) if 0 <= int(v) < V and float(l) != -math.inf]
        if not pairs or total == -math.inf:
            continue
        zs = torch.tensor([l for _, l in pairs]).double()
        q = torch.softmax(zs, 0)
        logq = torch.log_softmax(zs, 0)
        logp = (x[t] - m) - total
        g = logp.exp()
        for (v, _), qk, lq in zip(pairs, q, logq):
            if qk > 0:
                loss[t] += tau * tau * qk * (lq - logp[v])
                size[t] += tau * tau * qk * (2 + abs(lq) + abs(logp[v]))
            g[v] -= qk
        grad[t] = g * tau * (1.0 if weight is None else float(weight[t]))
    return loss, stats, grad, size


def logits_like(rows, V, seed, masked=0.0, empty=()):
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn((rows, V), generator=gen) * 2
    z.scatter_(1, torch.randint(0, V, (rows, 3), generator=gen), 6 + 3 * torch.randn((rows, 3), generator=gen))
    if masked:
        z[torch.rand((rows, V), generator=gen) < masked] = -math.inf
    for r in empty:
        z[r] = -math.inf
    return z
