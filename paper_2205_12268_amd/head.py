"""A class head on a WCC layer's maps, tuned for several customers at once, and what it answers: the operators on rows of tokens
together, as a program uses them.

A row is a pixel of the layer's output map, its channels last.  All images go through one frozen projection; each image's customer
has a low-rank adapter beside it.  The adapters are tuned by distillation from the teacher's best logits of every pixel
(``wcc_adapter_forward``, ``wcc_distill_forward`` with the gradient in place of the logits, ``wcc_adapter_backward``), then pixels
are answered with a class, its log probability, the entropy and the alternatives (``wcc_token_scores``).  With ``--block`` the maps go
through a trained block first (``block.GatedBlock``), which learns from the gradient of the head's input.

    python -m paper_2205_12268_amd.head [--steps 30] [--block]
"""
from __future__ import annotations

import argparse

import torch

from . import block, synth, wcc


class AdaptedHead:
    """Projection [classes, channels] in bf16, frozen, with adapters of one rank; fp32 masters of the adapters, bf16 copies for the
    kernels.  The context's workspace and the buffers are made once for `rows` rows."""

    def __init__(self, ctx: wcc.Context, w: torch.Tensor, adapters: int, rank: int, rows: int, teacher: int, temperature: float):
        self.ctx, self.w = ctx, w
        classes, channels = w.shape
        gen = torch.Generator().manual_seed(7)
        self.a = (torch.randn((adapters, rank, channels), generator=gen) / channels ** 0.5).to(w.device)
        self.b = torch.zeros((adapters, classes, rank), device=w.device)  # at first the projection alone
        self.desc = wcc.make_adapter_desc(rows, channels, classes, adapters, rank, wcc.BF16)
        self.loss_desc = wcc.make_distill_desc(rows, classes, teacher, wcc.BF16, wcc.F32, temperature)
        ctx.ensure_workspace(self.desc)
        ctx.ensure_workspace(self.loss_desc)
        self.logits = torch.empty((rows, classes), dtype=torch.bfloat16, device=w.device)
        self.loss = torch.empty(rows, device=w.device)
        self.weight = torch.full((rows,), 1.0 / rows, device=w.device)
        self.da, self.db = torch.empty_like(self.a), torch.empty_like(self.b)
        self._copies()

    def _copies(self):
        self.a16, self.b16 = self.a.bfloat16(), self.b.bfloat16()

    def project(self, x: torch.Tensor, adapter_of_row: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
        """Logits of any number of rows up to the head's own."""
        d = self.desc
        if x.shape[0] != d.rows:
            d = wcc.make_adapter_desc(x.shape[0], d.C_in, d.C_out, d.adapters, d.rank, wcc.BF16)
            self.ctx.ensure_workspace(d)
        self.ctx.wcc_adapter_forward(d, x, self.w, adapter_of_row, self.a16, self.b16, None, None, out)
        return out

    def step(self, x, adapter_of_row, t_idx, t_logit, rate: float, dx=None) -> torch.Tensor:
        """One step of gradient descent on the adapters; the losses of the rows before it, on the device.  dx: takes the gradient of x."""
        y = self.project(x, adapter_of_row, self.logits)
        self.ctx.wcc_distill_forward(self.loss_desc, y, t_idx, t_logit, self.loss, None, self.weight, y)  # y: its gradient now
        self.ctx.wcc_adapter_backward(self.desc, x, self.w, adapter_of_row, self.a16, self.b16, None, None, y, dx, self.da, self.db)
        self.a -= rate * self.da
        self.b -= rate * self.db
        self._copies()
        return self.loss

    def answer(self, x, adapter_of_row, classes, top: int):
        """(log probability of the given class, entropy, best classes, their log probabilities) of each row."""
        rows, dev = x.shape[0], x.device
        y = self.project(x, adapter_of_row, torch.empty((rows, self.desc.C_out), dtype=torch.bfloat16, device=dev))
        d = wcc.make_scores_desc(rows, self.desc.C_out, top, wcc.BF16)
        self.ctx.ensure_workspace(d)
        logprob, entropy = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        best, best_logprob = torch.empty((rows, top), dtype=torch.int32, device=dev), torch.empty((rows, top), device=dev)
        self.ctx.wcc_token_scores(d, y, classes, logprob, entropy, best, best_logprob)
        return logprob, entropy, best, best_logprob


def maps_of_a_layer(ctx: wcc.Context, images: int, channels: int, side: int) -> torch.Tensor:
    """Rows [images * side^2, channels] bf16: a WCC layer's output on synthetic maps, a pixel a row."""
    cfg = synth.small(synth.config(2), B=images, C_in=32, C_out=channels, H=side, W=side)
    x, w = synth.make_inputs(cfg)
    d = wcc.make_desc(cfg.B, cfg.C_in, cfg.C_out, cfg.H, cfg.W, cfg.levels, cfg.keep_num, cfg.keep_den, cfg.w_dtype, cfg.act_bits)
    ctx.ensure_workspace(d)
    y = torch.empty((images, channels, side, side), device="cuda")
    stored = torch.from_numpy(w.stored.view("int16")).cuda()
    ctx.wcc_forward(d, torch.from_numpy(x).cuda(), stored, None, 0.0, y)
    rows = y.permute(0, 2, 3, 1).reshape(-1, channels)
    return ((rows - rows.mean(dim=0)) / rows.std()).bfloat16().contiguous()


def demo(steps: int = 30, images: int = 4, side: int = 32, channels: int = 96, classes: int = 1000, rank: int = 8, teacher: int = 16,
         rate: float = 3.0, say=print, with_block: bool = False):
    """Losses of every step, and the answers to four pixels."""
    ctx = wcc.Context(0)
    rows = maps_of_a_layer(ctx, images, channels, side)
    n = rows.shape[0]
    gen = torch.Generator().manual_seed(5)
    w = (torch.randn((classes, channels), generator=gen) / channels ** 0.5).bfloat16().cuda()
    of_row = torch.arange(images, dtype=torch.int32, device="cuda").repeat_interleave(side * side)
    # the teacher: the projection with a hidden change for each customer, of which the best logits are kept
    hidden = torch.randn((images, classes, 4), generator=gen).cuda() @ torch.randn((images, 4, channels), generator=gen).cuda() / channels
    full = torch.cat([rows.view(images, -1, channels)[i].float() @ (w.float() + 2.0 * hidden[i]).t() for i in range(images)])
    t_logit, t_idx = full.topk(teacher, dim=1)
    t_logit, t_idx = t_logit.contiguous(), t_idx.int().contiguous()

    head = AdaptedHead(ctx, w, images, rank, n, teacher, temperature=2.0)
    front = block.GatedBlock(ctx, images, side * side, channels, 2 * channels, channels // 8) if with_block else None
    maps, dx = rows, torch.empty_like(rows) if front else None
    losses = []
    for i in range(steps):
        if front:
            rows = front.forward(maps)
        losses.append(float(head.step(rows, of_row, t_idx, t_logit, rate, dx).mean()))
        if front:
            front.backward(dx)
            front.step(rate / 3)
        if i % 10 == 0 or i == steps - 1:
            say(f"step {i}: loss {losses[-1]:.4f}")
    if front:
        rows = front.forward(maps)
    pick = torch.arange(images, device="cuda") * (side * side) + 5
    answers = head.answer(rows[pick], of_row[pick], t_idx[pick, 0].contiguous(), 3)
    torch.cuda.synchronize()
    for i, (lp, h, best, blp) in enumerate(zip(*[a.tolist() for a in answers])):
        say(f"customer {i}: log p of the teacher's class {lp:.3f}, entropy {h:.3f}, best " +
            ", ".join(f"{c} ({p:.3f})" for c, p in zip(best, blp)))
    ctx.close()
    return losses, answers, t_idx[pick]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--block", action="store_true", help="a trained block before the head")
    args = ap.parse_args()
    demo(args.steps, rate=1.0 if args.block else 3.0, with_block=args.block)
