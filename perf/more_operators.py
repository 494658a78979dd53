"""What the operators of a block on rows are timed on: activations kept in 8 bits, group norm with an activation on maps whose
channels come last, and the gated feed-forward block, each as a model's forward pass or a training step calls it.

All through the public binding ``paper_2205_12268_amd.wcc``:

* ``keep``        -- ``wcc_rows_keep``, ``wcc_rows_restore``: rows to 8 bits and back, as a layer does that keeps its input;
* ``norm``        -- ``wcc_group_norm_forward``;
* ``norm_train``  -- ``wcc_group_norm_forward`` and ``wcc_group_norm_backward``, with ``keep`` the input kept in 8 bits between them;
* ``gated``       -- ``wcc_gated_forward``;
* ``gated_train`` -- ``wcc_gated_forward`` and ``wcc_gated_backward``; ``keep`` "input": the input is kept in 8 bits between them,
  "all": the two projections too (else the backward pass makes them again), "none": the input stays as it is.

Types: "bf16" or "f32" for rows and weights; gamma, beta, their gradients and the statistics of groups are f32.
``pad``: elements between rows (a view of a wider buffer).  ``counts``: samples of a padded batch, of which a part of the pixels
is there.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_BLOCK = 32  # values of a row that share a step in 8 bits
_EPS = 1e-5


# --------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------
def _keep(name, rows, width, t="bf16", pad=0):
    return {"name": name, "kind": "keep", "rows": rows, "width": width, "type": t, "pad": pad}


def _norm(name, samples, pixels, C, groups, act, t="bf16", pad=0, counts=False, train=False, keep=False):
    return {"name": name, "kind": "norm_train" if train else "norm", "samples": samples, "pixels": pixels, "C": C, "groups": groups,
            "act": act, "type": t, "pad": pad, "counts": counts, "keep": keep}


def _gated(name, rows, ci, co, act, t="bf16", pad=0, train=False, keep="none"):
    return {"name": name, "kind": "gated_train" if train else "gated", "rows": rows, "C_in": ci, "C_out": co, "act": act, "type": t,
            "pad": pad, "keep": keep}


def listed():
    return [
        # the pixels of a layer's maps, kept for the backward pass of whatever reads them
        _keep("keep_maps", 131072, 256),
        # rows of odd width in fp32, views of a wider buffer
        _keep("keep_ragged_f32", 1777, 1001, t="f32", pad=3),
        # one small map, as in the deepest layer of a network that answers one image: latency
        _norm("norm_one_map", 1, 256, 96, 8, "silu"),
        # a batch of large maps: memory
        _norm("norm_maps", 8, 16384, 256, 32, "silu"),
        # a padded batch in groups of three channels, rows of a wider buffer
        _norm("norm_ragged_f32", 5, 1156, 96, 32, "relu", t="f32", pad=3, counts=True),
        # a training step on the batch of large maps, the input kept in 8 bits
        _norm("norm_train_kept", 8, 16384, 256, 32, "silu", train=True, keep=True),
        # the same on a backbone's expanded channels in fp32 and a padded batch, gelu
        _norm("norm_train_f32", 3, 1156, 960, 8, "gelu", t="f32", train=True, counts=True),
        # one token: what a serving loop pays at the least, the weights' bytes
        _gated("gated_one_token", 1, 2048, 5632, "silu"),
        # long prompts: the matrix cores
        _gated("gated_prompts", 8192, 2048, 8192, "silu"),
        # a short batch through sizes that nothing rounds, rows of a wider buffer
        _gated("gated_ragged", 777, 1000, 1537, "gelu", pad=3),
        # a training step that keeps everything in 8 bits
        _gated("gated_train_kept", 4096, 2048, 5632, "silu", train=True, keep="all"),
        # the same in fp32 on a backbone's expansion, 160 -> 960 channels, a pixel a row; the projections are made again
        _gated("gated_train_f32", 1156, 160, 960, "gelu", t="f32", train=True, keep="input"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["keep", "norm", "norm", "norm_train", "norm_train", "gated", "gated", "gated_train", "gated_train"])
    while True:
        t = rng.choice(["bf16", "bf16", "bf16", "f32"])
        pad = rng.choice([0, 0, 0, 8, 3])
        # (the slope of relu jumps at 0, of which two fp32 sums may lie on both sides; so training steps have the smooth ones here)
        act = rng.choice(["none", "silu", "silu", "gelu"] if kind.endswith("train") else ["none", "relu", "silu", "silu", "gelu"])
        if kind == "keep":
            case = _keep("", _log_int(rng, 1, 200000), _log_int(rng, 1, 8192), t, pad)
            dear = case["rows"] * (case["width"] + pad) > 131072 * 256
        elif kind.startswith("norm"):
            per = rng.choice([1, 2, 3, 4, 5, 8, 8, 8, 12, 16, 32, 120])  # channels of a group
            groups = _log_int(rng, 1, 64)
            case = _norm("", _log_int(rng, 1, 32), _log_int(rng, 1, 65536), per * groups, groups, act, t, pad, rng.random() < 0.3,
                         kind == "norm_train", kind == "norm_train" and rng.random() < 0.6)
            dear = case["samples"] * case["pixels"] * (case["C"] + pad) * _SIZE[t] > 8 * 16384 * 256 * 2
            dear = dear or case["pixels"] * per < 64  # (fewer values have no statistics to speak of: dx cancels to nothing)
        else:
            step = rng.choice([1, 8, 32, 64, 64])  # widths are mostly whole tiles, now and then not
            ci, co = (step * _log_int(rng, max(1, 64 // step), 8192 // step) for _ in range(2))
            train = kind == "gated_train"
            # (two fp32 sums of one projection may lie on both sides of a border between codes; so in fp32 only inputs are kept here)
            keep = rng.choice(["none", "input", "all", "all"] if t == "bf16" else ["none", "input"]) if train else "none"
            case = _gated("", _log_int(rng, 1, 8192), ci, co, act, t, pad, train, keep)
            dear = case["rows"] * ci * co * (3 if train else 1) > 8192 * 2048 * 8192
        if not dear:
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


def _room(rows, width, t, pad):
    return torch.zeros((rows, width + pad), dtype=_TORCH[t], device="cuda")[:, :width]


def _activations(gen, rows, width):
    """Rows as layers give them: channels of different sizes about means of their own, a few values far out."""
    x = _randn(gen, rows, width) * (0.3 + torch.rand(width, generator=gen, device="cuda")) + 0.5 * _randn(gen, width)
    far = torch.rand((rows, width), generator=gen, device="cuda") < 1e-3
    return torch.where(far, 20.0 * x, x)


def _prepare_keep(c, gen):
    rows, width, t, pad = c["rows"], c["width"], c["type"], c["pad"]
    blocks = -(-width // _BLOCK)
    return {"x": _rows(_activations(gen, rows, width), t, pad), "codes": torch.empty((rows, blocks * _BLOCK), dtype=torch.int8, device="cuda"),
            "steps": torch.empty((rows, blocks), dtype=torch.uint8, device="cuda"), "back": _room(rows, width, t, pad)}


def _prepare_norm(c, gen):
    n, p, ch, t, pad = c["samples"], c["pixels"], c["C"], c["type"], c["pad"]
    s = {"x": _rows(_activations(gen, n * p, ch), t, pad), "gamma": 1.0 + 0.2 * _randn(gen, ch), "beta": 0.2 * _randn(gen, ch),
         "y": _room(n * p, ch, t, pad), "counts": None}
    if c["counts"]:  # a padded batch: the first sample whole, and where there are several the last one empty
        counts = torch.randint(p // 2, p + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
        counts[0] = p
        if n > 2:
            counts[-1] = 0
        s["counts"] = counts
    if c["kind"] == "norm_train":
        s["stats"] = torch.empty((n, c["groups"], 2), device="cuda")
        s["dy"] = _rows(_randn(gen, n * p, ch) * 1e-2, t, pad)
        s["dx"] = _room(n * p, ch, t, pad)
        s["dgamma"], s["dbeta"] = torch.empty(ch, device="cuda"), torch.empty(ch, device="cuda")
        if c["keep"]:
            blocks = -(-ch // _BLOCK)
            s["codes"] = torch.empty((n * p, blocks * _BLOCK), dtype=torch.int8, device="cuda")
            s["steps"] = torch.empty((n * p, blocks), dtype=torch.uint8, device="cuda")
    return s


def _prepare_gated(c, gen):
    rows, ci, co, t, pad = c["rows"], c["C_in"], c["C_out"], c["type"], c["pad"]
    s = {"x": _rows(_activations(gen, rows, ci), t, pad),
         "w_gate": (_randn(gen, co, ci) / math.sqrt(ci)).to(_TORCH[t]), "w_up": (_randn(gen, co, ci) / math.sqrt(ci)).to(_TORCH[t]),
         "y": _room(rows, co, t, pad)}
    if c["kind"] == "gated_train":
        s["dy"] = _rows(_randn(gen, rows, co) * 1e-2, t, pad)
        s["dx"] = _room(rows, ci, t, pad)
        s["dw_gate"], s["dw_up"] = torch.empty_like(s["w_gate"]), torch.empty_like(s["w_up"])
        for name, width, lead in (("x", ci, ()), ("h", co, (2,))):
            if c["keep"] == "all" or (c["keep"] == "input" and name == "x"):
                blocks = -(-width // _BLOCK)
                s[name + "_codes"] = torch.empty((*lead, rows, blocks * _BLOCK), dtype=torch.int8, device="cuda")
                s[name + "_steps"] = torch.empty((*lead, rows, blocks), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"keep": _prepare_keep, "norm": _prepare_norm, "norm_train": _prepare_norm}.get(case["kind"], _prepare_gated)
    return {"case": case, **make(case, gen)}


# --------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------
def _kept(x):
    """What rows stand for once they are kept in 8 bits.  32 neighbours share a power of two, that of the largest of them over 64
    (twice that where the largest would round to 128, at least 2^-126); a value is the nearest multiple, ties to the even one."""
    rows, width = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -width % _BLOCK)).view(rows, -1, _BLOCK)
    top = v.abs().amax(dim=2, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top).exponent - 7, -126)
    e = e.clamp(min=-126)
    e = e + (top * _two(-e) >= 127.5)
    return ((v * _two(-e)).round() * _two(e)).view(rows, -1)[:, :width].to(x.dtype)


def _two(e):
    """2^e in 64 bits, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + (-z).exp())
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    """The derivative of _act."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + (-z).exp())
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * (-0.5 * z * z).exp() * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _grouped(s, rows):
    """[samples, pixels, groups, channels of a group] in fp32."""
    c = s["case"]
    return rows.float().reshape(c["samples"], c["pixels"], c["groups"], -1)


def _there(s):
    """Which pixels of the batch are there, [samples, pixels, 1, 1], and how many values a group has, [samples, 1, 1, 1]."""
    c = s["case"]
    counts = torch.full((c["samples"],), c["pixels"], device="cuda") if s["counts"] is None else s["counts"]
    mask = torch.arange(c["pixels"], device="cuda") < counts[:, None]
    return mask[:, :, None, None], (counts * (c["C"] // c["groups"])).clamp(min=1).float()[:, None, None, None]


def _plain_norm(s):
    c, (mask, size) = s["case"], _there(s)
    x = _grouped(s, s["x"])
    gamma, beta = s["gamma"].view(c["groups"], -1), s["beta"].view(c["groups"], -1)
    mean = torch.where(mask, x, 0.0).sum(dim=(1, 3), keepdim=True) / size
    var = torch.where(mask, (x - mean) ** 2, 0.0).sum(dim=(1, 3), keepdim=True) / size
    rstd = 1 / (var + _EPS).sqrt()
    shape, t = s["x"].shape, s["x"].dtype
    y = torch.where(mask, _act((x - mean) * rstd * gamma + beta, c["act"]), 0.0).reshape(shape).to(t)
    if c["kind"] == "norm":
        return y
    if c["keep"]:
        x = _grouped(s, _kept(s["x"]))
    xh = (x - mean) * rstd
    dz = torch.where(mask, _grouped(s, s["dy"]) * _slope(xh * gamma + beta, c["act"]), 0.0)
    dxh = dz * gamma
    m1 = dxh.sum(dim=(1, 3), keepdim=True) / size
    m2 = (dxh * xh).sum(dim=(1, 3), keepdim=True) / size
    dx = torch.where(mask, rstd * (dxh - m1 - xh * m2), 0.0).reshape(shape).to(t)
    return {"y": y, "dx": dx, "dgamma": (dz * xh).sum(dim=(0, 1)).reshape(-1), "dbeta": dz.sum(dim=(0, 1)).reshape(-1)}


def _plain_gated(s):
    c, t = s["case"], s["x"].dtype
    wg, wu, x = s["w_gate"].float(), s["w_up"].float(), s["x"].float()
    g, u = x @ wg.t(), x @ wu.t()
    y = (_act(g, c["act"]) * u).to(t)
    if c["kind"] == "gated":
        return y
    if c["keep"] != "none":
        x = _kept(s["x"]).float()
    if c["keep"] == "all":
        g, u = _kept(g), _kept(u)
    elif c["keep"] == "input":
        g, u = x @ wg.t(), x @ wu.t()
    dy = s["dy"].float()
    dg, du = dy * u * _slope(g, c["act"]), dy * _act(g, c["act"])
    return {"y": y, "dx": (dg @ wg + du @ wu).to(t), "dw_gate": (dg.t() @ x).to(t), "dw_up": (du.t() @ x).to(t)}


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
    if c["kind"] == "keep":
        return wcc.make_rows_desc(c["rows"], c["width"], t, ld=c["width"] + c["pad"])
    act = {"none": wcc.ACT_NONE, "relu": wcc.ACT_RELU, "silu": wcc.ACT_SILU, "gelu": wcc.ACT_GELU}[c["act"]]
    if c["kind"].startswith("norm"):
        desc = wcc.make_group_norm_desc(c["samples"], c["pixels"], c["C"], c["groups"], t, act, _EPS, ldx=c["C"] + c["pad"],
                                        ldy=c["C"] + c["pad"])
    else:
        desc = wcc.make_gated_desc(c["rows"], c["C_in"], c["C_out"], t, act, train=c["kind"] == "gated_train", ldx=c["C_in"] + c["pad"],
                                   ldy=c["C_out"] + c["pad"])
        s["rows_desc"] = wcc.make_rows_desc(c["rows"], c["C_in"], t, ld=c["C_in"] + c["pad"])
    _ctx[0].ensure_workspace(desc)
    return desc


def _own(s):
    if "desc" not in s:
        s["desc"] = _plan(s)
    ctx, d, c = _ctx[0], s["desc"], s["case"]
    if c["kind"] == "keep":
        ctx.wcc_rows_keep(d, s["x"], s["codes"], s["steps"])
        ctx.wcc_rows_restore(d, s["codes"], s["steps"], s["back"])
        return s["back"]
    if c["kind"].startswith("norm"):
        kept = (s.get("codes"), s.get("steps"))
        ctx.wcc_group_norm_forward(d, s["x"], s["gamma"], s["beta"], s["counts"], s["y"], s.get("stats"), *kept)
        if c["kind"] == "norm":
            return s["y"]
        ctx.wcc_group_norm_backward(d, None if c["keep"] else s["x"], *kept, s["gamma"], s["beta"], s["counts"], s["stats"], s["dy"],
                                    s["dx"], s["dgamma"], s["dbeta"])
        return {k: s[k] for k in ("y", "dx", "dgamma", "dbeta")}
    hidden = (s.get("h_codes"), s.get("h_steps"))
    if "x_codes" in s:
        ctx.wcc_rows_keep(s["rows_desc"], s["x"], s["x_codes"], s["x_steps"])
    ctx.wcc_gated_forward(d, s["x"], s["w_gate"], s["w_up"], s["y"], *hidden)
    if c["kind"] == "gated":
        return s["y"]
    ctx.wcc_gated_backward(d, None if "x_codes" in s else s["x"], s.get("x_codes"), s.get("x_steps"), s["w_gate"], s["w_up"], *hidden,
                           s["dy"], s["dx"], s["dw_gate"], s["dw_up"])
    return {k: s[k] for k in ("y", "dx", "dw_gate", "dw_up")}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return _kept(state["x"]) if kind == "keep" else _plain_norm(state) if kind.startswith("norm") else _plain_gated(state)


# --------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------
def work(case):
    c, size = case, _SIZE[case["type"]]
    if c["kind"] == "keep":  # x in, the values out; the codes written and read between
        n = c["rows"] * c["width"]
        return {"bytes": int(n * (2 * size + 2 * 33 / 32)), "flops": 4 * n}
    if c["kind"].startswith("norm"):
        n = c["samples"] * c["pixels"] * c["C"]
        if c["kind"] == "norm":
            return {"bytes": n * 2 * size, "flops": 10 * n}
        # x in, y out, dy in, dx out; between the passes the codes, or x again
        return {"bytes": int(n * (4 * size + (2 * 33 / 32 if c["keep"] else size))), "flops": 30 * n}
    rows, ci, co = c["rows"], c["C_in"], c["C_out"]
    product = 4 * rows * ci * co  # both projections
    if c["kind"] == "gated":
        return {"bytes": size * (rows * (ci + co) + 2 * ci * co), "flops": product}
    kept = rows * (2 * 33 / 32) * {"none": 0, "input": ci, "all": ci + 2 * co}[c["keep"]]
    again = rows * ci * size if c["keep"] == "none" else 0
    # x, both weights, dy in; y, dx, both gradients out.  Projections (made again unless kept), dx, the weights' gradients
    return {"bytes": int(size * (rows * 2 * (ci + co) + 4 * ci * co) + kept + again), "flops": product * (3 if c["keep"] == "all" else 4)}


# --------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------
def _exact_kept(x):
    """In whole steps of each block's own size, found by comparison rather than from the bits of its largest value."""
    rows, width = x.shape
    out = torch.zeros((rows, -(-width // _BLOCK) * _BLOCK), dtype=torch.float64, device="cuda")
    out[:, :width] = x
    out = out.view(-1, _BLOCK)
    limit = out.abs().max(dim=1).values
    # the first of the steps 2^-126, 2^-125, ... of which 127.5 exceed the block's largest: no code is beyond 127
    steps = torch.tensor([2.0 ** e for e in range(-126, 123)], dtype=torch.float64, device="cuda")
    step = steps[torch.searchsorted(127.5 * steps, limit, right=True)][:, None]
    return (torch.round(out / step) * step).view(rows, -1)[:, :width]


def _exact_act(z, act):
    """(value, derivative)"""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    below = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _exact_norm(s):
    """Sample by sample, on the pixels that are there."""
    c = s["case"]
    n, p, groups, train = c["samples"], c["pixels"], c["groups"], c["kind"] == "norm_train"
    out = {k: torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda") for k in (("y", "dx") if train else ("y",))}
    dgamma = torch.zeros(c["C"], dtype=torch.float64, device="cuda")
    dbeta = torch.zeros_like(dgamma)
    gamma, beta = s["gamma"].double(), s["beta"].double()
    counts = [p] * n if s["counts"] is None else s["counts"].tolist()
    for i, m in enumerate(counts):
        if m == 0:
            continue
        at = slice(i * p, i * p + m)
        by_group = lambda v: v.reshape(m, groups, -1).transpose(0, 1).reshape(groups, -1)  # noqa: E731
        to_rows = lambda v: v.reshape(groups, m, -1).transpose(0, 1).reshape(m, -1)  # noqa: E731
        x = by_group(s["x"][at].double())
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = torch.rsqrt(var + _EPS)
        out["y"][at] = _exact_act(to_rows((x - mean) * rstd) * gamma + beta, c["act"])[0]
        if not train:
            continue
        if c["keep"]:
            x = by_group(_exact_kept(s["x"][at]))
        xh = (x - mean) * rstd
        dz = s["dy"][at].double() * _exact_act(to_rows(xh) * gamma + beta, c["act"])[1]
        dgamma += (dz * to_rows(xh)).sum(dim=0)
        dbeta += dz.sum(dim=0)
        d = by_group(dz * gamma)
        out["dx"][at] = to_rows(rstd * (d - d.mean(dim=1, keepdim=True) - xh * (d * xh).mean(dim=1, keepdim=True)))
    return {**out, "dgamma": dgamma, "dbeta": dbeta} if train else out["y"]


def _exact_gated(s):
    c = s["case"]
    both = torch.cat([s["w_gate"], s["w_up"]]).double()
    x = s["x"].double()
    g, u = (x @ both.t()).chunk(2, dim=1)
    y = _exact_act(g, c["act"])[0] * u
    if c["kind"] == "gated":
        return y
    if c["keep"] != "none":
        x = _exact_kept(s["x"])
        g, u = (_exact_kept(g), _exact_kept(u)) if c["keep"] == "all" else (x @ both.t()).chunk(2, dim=1)
    value, slope = _exact_act(g, c["act"])
    dy = s["dy"].double()
    d = torch.cat([dy * u * slope, dy * value], dim=1)
    dw = d.t() @ x
    return {"y": y, "dx": d @ both, "dw_gate": dw[:c["C_out"]], "dw_up": dw[c["C_out"]:]}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_kept(s["x"]) if case["kind"] == "keep" else _exact_norm(s) if case["kind"].startswith("norm") else _exact_gated(s)
