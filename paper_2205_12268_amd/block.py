"""A block on a layer's maps that can be trained: group norm with an activation, the gated feed-forward block, a frozen projection back
and the sum with its input.  A row is a pixel of the maps, its channels last.

Between the passes the block holds 8-bit rows only: its input, the normalised rows and the two projections (``wcc_group_norm_forward``
and ``wcc_gated_forward`` keep them as they go, ``wcc_rows_keep`` the rows between); the backward pass reads them.
"""
from __future__ import annotations

import torch

from . import wcc


def _kept(*shape, device):
    room = wcc.kept_room(shape[-1])
    return (torch.empty((*shape[:-1], room), dtype=torch.int8, device=device),
            torch.empty((*shape[:-1], room // wcc.KEPT_BLOCK), dtype=torch.uint8, device=device))


class GatedBlock:
    """For `samples` maps of `pixels` pixels, in bf16; fp32 masters of its weights, bf16 copies for the kernels.  Made once, with the
    context's workspace and all buffers."""

    def __init__(self, ctx: wcc.Context, samples: int, pixels: int, channels: int, hidden: int, groups: int, device="cuda", seed: int = 11):
        self.ctx, rows = ctx, samples * pixels
        gen = torch.Generator().manual_seed(seed)
        draw = lambda n, k, size: (torch.randn((n, k), generator=gen) * size / k ** 0.5).to(device)  # noqa: E731
        self.masters = {"gamma": torch.ones(channels, device=device), "beta": torch.zeros(channels, device=device),
                        "w_gate": draw(hidden, channels, 1.0), "w_up": draw(hidden, channels, 1.0)}
        self.w_down = draw(channels, hidden, 0.1).bfloat16()  # (at first the maps all but as they are)
        self.norm = wcc.make_group_norm_desc(samples, pixels, channels, groups, wcc.BF16, wcc.ACT_SILU)
        self.rows = wcc.make_rows_desc(rows, channels, wcc.BF16)
        self.gated = wcc.make_gated_desc(rows, channels, hidden, wcc.BF16, wcc.ACT_SILU, train=True)
        self.down = wcc.make_adapter_desc(rows, hidden, channels, 0, 0, wcc.BF16)
        for d in (self.norm, self.gated, self.down):
            ctx.ensure_workspace(d)
        buffer = lambda width: torch.empty((rows, width), dtype=torch.bfloat16, device=device)  # noqa: E731
        self.n, self.h, self.out, self.dh, self.dn, self.dx = (buffer(w) for w in (channels, hidden, channels, hidden, channels, channels))
        self.stats = torch.empty((samples, groups, 2), device=device)
        self.x_kept, self.n_kept = _kept(rows, channels, device=device), _kept(rows, channels, device=device)
        self.h_kept = _kept(2, rows, hidden, device=device)
        self.grads = {"gamma": torch.empty(channels, device=device), "beta": torch.empty(channels, device=device),
                      "w_gate": torch.empty((hidden, channels), dtype=torch.bfloat16, device=device),
                      "w_up": torch.empty((hidden, channels), dtype=torch.bfloat16, device=device)}
        self._copies()

    def _copies(self):
        self.w_gate, self.w_up = self.masters["w_gate"].bfloat16(), self.masters["w_up"].bfloat16()

    def forward(self, x: torch.Tensor, counts=None) -> torch.Tensor:
        """x + W_down (silu(W_gate n) * W_up n), n = silu(group norm of x); rows that `counts` leaves out stay x."""
        ctx, m = self.ctx, self.masters
        if counts is not None:
            self.n.zero_()  # (rows that are not there stay as they are: nothing, for the products)
        ctx.wcc_group_norm_forward(self.norm, x, m["gamma"], m["beta"], counts, self.n, self.stats, *self.x_kept)
        ctx.wcc_rows_keep(self.rows, self.n, *self.n_kept)
        ctx.wcc_gated_forward(self.gated, self.n, self.w_gate, self.w_up, self.h, *self.h_kept)
        ctx.wcc_adapter_forward(self.down, self.h, self.w_down, None, None, None, None, None, self.out)
        self.out += x
        return self.out

    def backward(self, dout: torch.Tensor, counts=None) -> torch.Tensor:
        """The gradient of the input for a gradient of the output; those of the weights are left in `grads`.  Rows that `counts` leaves out
        take part in them with an input of 0, so `dout` has to be finite there too."""
        ctx, m, g = self.ctx, self.masters, self.grads
        ctx.wcc_adapter_backward(self.down, None, self.w_down, None, None, None, None, None, dout, self.dh)
        ctx.wcc_gated_backward(self.gated, None, *self.n_kept, self.w_gate, self.w_up, *self.h_kept, self.dh, self.dn, g["w_gate"], g["w_up"])
        if counts is not None:
            self.dx.zero_()
        ctx.wcc_group_norm_backward(self.norm, None, *self.x_kept, m["gamma"], m["beta"], counts, self.stats, self.dn, self.dx, g["gamma"],
                                    g["beta"])
        self.dx += dout
        return self.dx

    def step(self, rate: float) -> None:
        """One step of gradient descent by the gradients of the last backward pass."""
        for k, v in self.masters.items():
            v -= rate * self.grads[k].float()
        self._copies()
