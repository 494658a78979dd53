"""What the operators of a model's head are timed on: the projection with low-rank adapters, the scores of its logits, and the
distillation loss.

Three families, all through the public binding ``paper_2205_12268_amd.wcc``:

* ``adapter``, ``adapter_grad`` -- ``wcc_adapter_forward`` / ``wcc_adapter_backward``: one shared projection over the tokens of
  many requests, beside it the low-rank adapter of each token's request;
* ``scores``  -- ``wcc_token_scores``: log probability of a given token, entropy and the top alternatives of each row of logits;
* ``distill`` -- ``wcc_distill_forward`` / ``wcc_distill_backward``: the divergence from a teacher of which the top logits are
  kept; ``mode`` says whether the loss alone, the gradient alone or both in one call ("step") are asked for.

Types: "bf16" or "f32" for activations, weights and logits; row statistics, losses and the adapters' gradients are f32.
``pad``: elements between the rows of the activations or logits (a view of a wider buffer).
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}


# --------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------
def _adapter(name, rows, ci, co, adapters, rank, order, t="bf16", pad=0, grad=False):
    return {"name": name, "kind": "adapter_grad" if grad else "adapter", "rows": rows, "C_in": ci, "C_out": co,
            "adapters": adapters, "rank": rank, "order": order, "type": t, "pad": pad}


def _scores(name, rows, V, top, t="bf16", pad=0, masked=0.0):
    return {"name": name, "kind": "scores", "rows": rows, "V": V, "top": top, "type": t, "pad": pad, "masked": masked}


def _distill(name, mode, rows, V, K, tau, t="bf16", pad=0, masked=0.0):
    return {"name": name, "kind": "distill", "mode": mode, "rows": rows, "V": V, "K": K, "tau": tau, "type": t, "pad": pad,
            "masked": masked}


def listed():
    return [
        # one token of one request: what a serving loop pays at the least
        _adapter("adapter_one_token", 1, 2048, 2048, 8, 16, "mixed"),
        # a decoding step: a token each of 32 requests, most with an adapter of their own
        _adapter("adapter_decode_32", 32, 4096, 4096, 24, 16, "mixed"),
        # a short batch of prompts through sizes that nothing rounds, rows of a wider buffer
        _adapter("adapter_ragged", 777, 1000, 1537, 5, 24, "runs", pad=3),
        # long prompts of several requests at once: bound by the matrix cores
        _adapter("adapter_prompts", 8192, 4096, 4096, 8, 32, "runs"),
        # a training step of four adapters on one batch: the projection is frozen, its input has a gradient
        _adapter("adapter_train", 4096, 2048, 4096, 4, 16, "runs", grad=True),
        # the same in fp32 on a backbone's expansion, 160 -> 960 channels, a pixel a row
        _adapter("adapter_train_f32", 1156, 160, 960, 3, 8, "runs", t="f32", grad=True),
        # the answer of one decoding step: a single row, which one compute unit would take long to read
        _scores("scores_one_row", 1, 131072, 20),
        # a batch whose vocabulary fits no tile, a tenth of it masked
        _scores("scores_batch_f32", 200, 50001, 5, t="f32", masked=0.1),
        # scoring whole prompts
        _scores("scores_prompts", 4096, 32768, 8),
        # a training step on the teacher's 64 best: loss and gradient in one call
        _distill("distill_step", "step", 4096, 65536, 64, 2.0),
        # the same at odd sizes in fp32 with masked logits, short teacher lists and rows without any
        _distill("distill_step_ragged_f32", "step", 333, 30011, 17, 1.5, t="f32", pad=5, masked=0.1),
        # the gradient by itself, as automatic differentiation asks for it
        _distill("distill_backward", "backward", 1000, 131072, 32, 1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["adapter", "adapter", "adapter", "adapter_grad", "adapter_grad", "scores", "scores", "distill", "distill"])
    while True:
        t = rng.choice(["bf16", "bf16", "bf16", "f32"])
        pad = rng.choice([0, 0, 0, 8, 3])
        if kind.startswith("adapter"):
            step = rng.choice([1, 8, 32, 64, 64])  # widths are mostly whole tiles, now and then not
            ci, co = (step * _log_int(rng, max(1, 64 // step), 6144 // step) for _ in range(2))
            case = _adapter("", _log_int(rng, 1, 8192), ci, co, _log_int(rng, 1, 32), rng.choice([1, 4, 8, 8, 16, 16, 24, 32, 64]),
                            rng.choice(["runs", "mixed"]), t, pad, kind == "adapter_grad")
            # no dearer than the longest prompts listed, the plain form's time included
            dear = case["rows"] * ci * co > 8192 * 4096 * 4096 or case["adapters"] * case["rank"] > 512
        else:
            rows, V = _log_int(rng, 1, 8192), _log_int(rng, 1000, 200000)
            masked = rng.choice([0.0, 0.0, 0.1, 0.9])
            if kind == "scores":
                case = _scores("", rows, V, rng.choice([0, 1, 5, 8, 20, 50]), t, pad, masked)
            else:
                case = _distill("", rng.choice(["loss", "step", "step", "backward"]), rows, V, _log_int(rng, 1, 128),
                                rng.choice([1.0, 1.0, 2.0, 4.0]), t, pad, masked)
            dear = rows * V > 4096 * 65536 // (2 if t == "f32" else 1)
        if not dear and 3072 not in case.values():
            del case["name"]
            return case


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows(values, t, pad):
    """`values` in type `t`, each row `pad` elements apart from the next."""
    rows, width = values.shape
    buf = torch.zeros((rows, width + pad), dtype=_TORCH[t], device="cuda")
    buf[:, :width] = values
    return buf[:, :width]


def _empty_rows(rows, width, t, pad):
    return torch.empty((rows, width + pad), dtype=_TORCH[t], device="cuda")[:, :width]


def _prepare_adapter(c, gen):
    rows, ci, co, n, r, t = c["rows"], c["C_in"], c["C_out"], c["adapters"], c["rank"], c["type"]
    if c["order"] == "mixed":  # any request's token in any row, one in eight without an adapter
        of_row = torch.randint(0, n, (rows,), generator=gen, device="cuda")
        of_row[torch.rand(rows, generator=gen, device="cuda") < 0.125] = -1
        of_row[0] = n - 1
    else:  # the prompts of the requests one after the other, in lengths that nothing rounds
        cuts = torch.rand(2 * n - 1, generator=gen, device="cuda").sort().values * rows
        request = torch.bucketize(torch.arange(rows, device="cuda").float(), cuts)
        whose = torch.cat([torch.randperm(n, generator=gen, device="cuda"), torch.randint(-1, n, (n,), generator=gen, device="cuda")])
        of_row = whose[request]
    low = max(1, r // 2)
    s = {
        "x": _rows(_randn(gen, rows, ci), t, c["pad"]),
        "w": (_randn(gen, co, ci) / math.sqrt(ci)).to(_TORCH[t]),
        "of_row": of_row.to(torch.int32),
        "a": (_randn(gen, n, r, ci) / math.sqrt(ci)).to(_TORCH[t]),
        "b": (_randn(gen, n, co, r) * (0.2 / math.sqrt(r))).to(_TORCH[t]),
        "ranks": torch.randint(low, r + 1, (n,), generator=gen, device="cuda", dtype=torch.int32),
        "scale": 0.5 + 1.5 * torch.rand(n, generator=gen, device="cuda"),
    }
    if c["kind"] == "adapter_grad":
        s["dy"] = _rows(_randn(gen, rows, co) * 1e-2, t, c["pad"])
        s["dx"] = _empty_rows(rows, ci, t, c["pad"])
        s["da"] = torch.empty((n, r, ci), dtype=torch.float32, device="cuda")
        s["db"] = torch.empty((n, co, r), dtype=torch.float32, device="cuda")
    else:
        s["y"] = _empty_rows(rows, co, t, c["pad"])
    return s


def _logits(c, gen):
    """Rows as a trained head gives them: a wide bulk and a few tokens far above it, in some cases masked tokens."""
    rows, V = c["rows"], c["V"]
    z = _randn(gen, rows, V) * 2.0
    peaks = torch.randint(0, V, (rows, 8), generator=gen, device="cuda")
    z.scatter_(1, peaks, 6.0 + 3.0 * _randn(gen, rows, 8))
    if c["masked"]:
        z[torch.rand((rows, V), generator=gen, device="cuda") < c["masked"]] = -math.inf
        if rows > 4:  # a row in which the mask leaves nothing
            z[rows // 2] = -math.inf
    return _rows(z, c["type"], c["pad"])


def _prepare_scores(c, gen):
    rows, top = c["rows"], c["top"]
    s = {"logits": _logits(c, gen)}
    s["tokens"] = torch.randint(0, c["V"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
    s["logprob"], s["entropy"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s["top_idx"] = torch.empty((rows, top), dtype=torch.int32, device="cuda")
    s["top_logprob"] = torch.empty((rows, top), device="cuda")
    return s


def _prepare_distill(c, gen):
    rows, V, K = c["rows"], c["V"], min(c["K"], c["V"])
    s = {"logits": _logits(c, gen)}
    # the teacher's best: distinct tokens, a stride apart from a start of the row's own, logits falling
    start = torch.randint(0, V, (rows, 1), generator=gen, device="cuda")
    idx = (start + (V // K) * torch.arange(K, device="cuda")) % V
    z = _randn(gen, rows, K).mul_(2.0).add_(4.0).sort(dim=1, descending=True).values
    if c["masked"]:
        count = torch.randint(1, K + 1, (rows, 1), generator=gen, device="cuda")
        if rows > 6:
            count[rows // 3] = 0  # a row without a teacher
        idx = torch.where(torch.arange(K, device="cuda") < count, idx, -1)
        # what a mask hides from the student the teacher does not propose, but in a row that has nothing left
        seen = s["logits"].float().gather(1, idx.clamp(min=0)) > -math.inf
        idx = torch.where(seen, idx, -1)
    s["t_idx"], s["t_logit"] = idx.to(torch.int32).contiguous(), z.contiguous()
    s["weight"] = torch.rand(rows, generator=gen, device="cuda") / rows
    s["loss"], s["stats"] = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    if c["mode"] == "backward":  # what the forward call left: a row's largest logit, and the log of its sum beside it
        x = s["logits"].float() / c["tau"]
        m = x.amax(dim=1)
        s["stats"] = torch.stack([m, (x - torch.where(m == -math.inf, 0.0, m)[:, None]).exp().sum(dim=1).log()], dim=1)
    if c["mode"] != "loss":
        s["dlogits"] = _empty_rows(rows, V, c["type"], c["pad"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"scores": _prepare_scores, "distill": _prepare_distill}.get(case["kind"], _prepare_adapter)
    return {"case": case, **make(case, gen)}


# --------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------
def _flat(s):
    """The adapters side by side: A [n r, C_in], B [n r, C_out], and the factor [rows, n r] that a row has for each line."""
    n, r, ci = s["a"].shape
    j, line = torch.arange(r, device="cuda"), torch.arange(n, device="cuda")
    factor = torch.where(j < s["ranks"][:, None], s["scale"][:, None], 0.0).reshape(-1)
    mine = s["of_row"][:, None] == line.repeat_interleave(r)
    return s["a"].float().reshape(n * r, ci), s["b"].float().transpose(1, 2).reshape(n * r, -1), mine * factor


def _plain_adapter(s):
    a, b, f = _flat(s)
    x = s["x"].float()
    return (x @ s["w"].float().t() + (x @ a.t() * f) @ b).to(s["x"].dtype)


def _plain_adapter_grad(s):
    a, b, f = _flat(s)
    x, dy = s["x"].float(), s["dy"].float()
    h, g = x @ a.t() * f, dy @ b.t() * f
    n, r, ci = s["a"].shape
    return {"dx": (dy @ s["w"].float() + g @ a).to(s["x"].dtype), "da": (g.t() @ x).reshape(n, r, ci),
            "db": (h.t() @ dy).reshape(n, r, -1).transpose(1, 2).contiguous()}


def _log_p(x):
    """(log p, [largest, log of the sum of exp(x - largest)]) of rows in fp32; -inf throughout where a row holds nothing else."""
    top = x.amax(dim=1, keepdim=True)
    m = torch.where(top == -math.inf, 0.0, top)
    log_total = (x - m).exp().sum(dim=1, keepdim=True).log()
    return torch.where(x == -math.inf, -math.inf, (x - m) - log_total), torch.cat([top, log_total], dim=1)


def _plain_scores(s):
    x = s["logits"].float()
    logp, _ = _log_p(x)
    p = logp.exp()
    order = x.sort(dim=1, descending=True, stable=True).indices[:, :s["case"]["top"]]
    return {"logprob": logp.gather(1, s["tokens"][:, None].long())[:, 0],
            "entropy": -(torch.where(p > 0, p * logp, 0.0)).sum(dim=1),
            "top_idx": order.to(torch.int32), "top_logprob": logp.gather(1, order)}


def _teacher(s, tau):
    """(q, log q, token, whether there is any) of the teacher's entries, in fp32."""
    there = s["t_idx"] >= 0
    z = torch.where(there, s["t_logit"] / tau, -math.inf)
    logq, stats = _log_p(z)
    return logq.exp(), torch.where(there, logq, 0.0), s["t_idx"].clamp(min=0).long(), stats[:, 1:] > -math.inf


def _plain_gradient(s, p, q, at, live):
    grad = p.scatter_add(1, at, -q) * (s["weight"] * s["case"]["tau"])[:, None]
    return torch.where(live, grad, 0.0).to(s["logits"].dtype)


def _plain_distill(s):
    tau, mode = s["case"]["tau"], s["case"]["mode"]
    x = s["logits"].float() / tau
    q, logq, at, live = _teacher(s, tau)
    if mode == "backward":
        m, log_total = s["stats"][:, :1], s["stats"][:, 1:]
        return {"dlogits": _plain_gradient(s, ((x - m) - log_total).exp(), q, at, live & (log_total > -math.inf))}
    logp, stats = _log_p(x)
    live = live & (stats[:, 1:] > -math.inf)
    each = torch.where(live & (q > 0), q * (logq - logp.gather(1, at)), 0.0)
    out = {"loss": tau * tau * each.sum(dim=1), "stats": stats}
    if mode == "step":
        out["dlogits"] = _plain_gradient(s, logp.exp(), q, at, live)
    return out


# --------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------
_ctx = []  # the one context of the program


def _plan(s):
    """What a program makes once and keeps beside its buffers: the descriptor, and a workspace large enough for it."""
    from paper_2205_12268_amd import wcc

    c = s["case"]
    t = {"bf16": wcc.BF16, "f32": wcc.F32}[c["type"]]
    if not _ctx:
        _ctx.append(wcc.Context(0))
    if c["kind"] == "scores":
        desc = wcc.make_scores_desc(c["rows"], c["V"], c["top"], t, ld=c["V"] + c["pad"])
    elif c["kind"] == "distill":
        desc = wcc.make_distill_desc(c["rows"], c["V"], s["t_idx"].shape[1], t, wcc.F32, c["tau"], ld=c["V"] + c["pad"],
                                     ld_grad=c["V"] + c["pad"])
    else:
        desc = wcc.make_adapter_desc(c["rows"], c["C_in"], c["C_out"], c["adapters"], c["rank"], t, ldx=c["C_in"] + c["pad"],
                                     ldy=c["C_out"] + c["pad"])
    _ctx[0].ensure_workspace(desc)
    return desc


def _own(s):
    if "desc" not in s:
        s["desc"] = _plan(s)
    ctx, d, kind = _ctx[0], s["desc"], s["case"]["kind"]
    if kind == "adapter":
        ctx.wcc_adapter_forward(d, s["x"], s["w"], s["of_row"], s["a"], s["b"], s["ranks"], s["scale"], s["y"])
        return s["y"]
    if kind == "adapter_grad":
        ctx.wcc_adapter_backward(d, s["x"], s["w"], s["of_row"], s["a"], s["b"], s["ranks"], s["scale"], s["dy"], s["dx"], s["da"],
                                 s["db"])
        return {"dx": s["dx"], "da": s["da"], "db": s["db"]}
    if kind == "scores":
        ctx.wcc_token_scores(d, s["logits"], s["tokens"], s["logprob"], s["entropy"], s["top_idx"], s["top_logprob"])
        return {k: s[k] for k in ("logprob", "entropy", "top_idx", "top_logprob")}
    if s["case"]["mode"] == "backward":
        ctx.wcc_distill_backward(d, s["logits"], s["t_idx"], s["t_logit"], s["stats"], s["weight"], s["dlogits"])
        return {"dlogits": s["dlogits"]}
    ctx.wcc_distill_forward(d, s["logits"], s["t_idx"], s["t_logit"], s["loss"], s["stats"], s["weight"], s.get("dlogits"))
    return {k: s[k] for k in ("loss", "stats", "dlogits") if k in s}


def run(state):
    if own:
        return _own(state)
    plain = {"adapter": _plain_adapter, "adapter_grad": _plain_adapter_grad, "scores": _plain_scores, "distill": _plain_distill}
    return plain[state["case"]["kind"]](state)


# --------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------
def work(case):
    c, size = case, _SIZE[case["type"]]
    rows = c["rows"]
    if c["kind"] in ("adapter", "adapter_grad"):
        ci, co, r = c["C_in"], c["C_out"], c["rank"]
        used = min(c["adapters"], rows) * r * (ci + co)
        low = 2 * rows * r * (ci + co)
        if c["kind"] == "adapter":
            return {"bytes": size * (rows * (ci + co) + ci * co + used) + 4 * rows, "flops": 2 * rows * ci * co + low}
        # x, dy, W, A, B in; dx, dA, dB out.  Products: W^T dy; h and g; A^T g, dA and dB
        return {"bytes": size * (rows * (2 * ci + co) + ci * co + used) + 4 * c["adapters"] * r * (ci + co) + 4 * rows,
                "flops": 2 * rows * ci * co + 2 * low + 2 * rows * r * ci}
    n = rows * c["V"]
    if c["kind"] == "scores":
        return {"bytes": n * size + rows * (12 + 8 * c["top"]), "flops": 5 * n}
    grad = c["mode"] != "loss"
    return {"bytes": n * size * (2 if grad else 1) + rows * (20 + 8 * c["K"]), "flops": (6 if grad else 4) * n}


# --------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------
def _exact_adapter(s):
    x, w = s["x"].double(), s["w"].double()
    grad = "dy" in s
    top = s["dy"].double() if grad else None
    y = None if grad else x @ w.t()
    dx = top @ w if grad else None
    da, db = [], []
    for i in range(s["a"].shape[0]):
        at = (s["of_row"] == i).nonzero()[:, 0]
        r, f = int(s["ranks"][i]), float(s["scale"][i])
        a, b = s["a"][i, :r].double(), s["b"][i, :, :r].double()
        if not grad:
            y[at] += f * ((x[at] @ a.t()) @ b.t())
            continue
        gy = top[at] @ b
        dx[at] += f * (gy @ a)
        da.append(torch.zeros(s["a"].shape[1:], dtype=torch.float64, device="cuda"))
        db.append(torch.zeros(s["b"].shape[1:], dtype=torch.float64, device="cuda"))
        da[-1][:r] = f * (gy.t() @ x[at])
        db[-1][:, :r] = f * (top[at].t() @ (x[at] @ a.t()))
    return {"dx": dx, "da": torch.stack(da), "db": torch.stack(db)} if grad else y


def _exact_scores(s):
    x, top = s["logits"].double(), s["case"]["top"]
    lse = torch.logsumexp(x, dim=1)
    dead = lse == -math.inf
    weight = torch.softmax(x, dim=1)
    mean = (weight * torch.where(x == -math.inf, 0.0, x)).sum(dim=1)
    best = x.sort(dim=1, descending=True).values[:, :top]
    given = x[torch.arange(len(x), device="cuda"), s["tokens"].long()]
    return {"logprob": torch.where(dead, -math.inf, given - lse), "entropy": torch.where(dead, 0.0, lse - mean), "top_idx": None,
            "top_logprob": torch.where(dead[:, None], -math.inf, best - lse[:, None])}


def _exact_distill(s):
    c = s["case"]
    tau, mode = c["tau"], c["mode"]
    x = s["logits"].double() / tau
    lse = s["stats"].double().sum(dim=1) if mode == "backward" else torch.logsumexp(x, dim=1)
    there = s["t_idx"] >= 0
    live = there.any(dim=1) & (lse > -math.inf)
    q = torch.softmax(torch.where(there, s["t_logit"].double() / tau, -math.inf), dim=1)
    q = torch.where(there & live[:, None], q, 0.0)
    at = s["t_idx"].clamp(min=0).long()
    out = {}
    if mode != "backward":
        picked = torch.where(q > 0, x.gather(1, at) - lse[:, None], 0.0)
        best = x.max(dim=1).values
        out = {"loss": tau ** 2 * (torch.special.xlogy(q, q) - q * picked).sum(dim=1),
               "stats": torch.stack([best, torch.where(best == -math.inf, -math.inf, lse - best)], dim=1)}
    if mode != "loss":
        p = torch.exp(x - lse[:, None])
        p.scatter_add_(1, at, -q)
        out["dlogits"] = torch.where(live[:, None], p * (tau * s["weight"].double())[:, None], 0.0)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return {"scores": _exact_scores, "distill": _exact_distill}.get(case["kind"], _exact_adapter)(state)
