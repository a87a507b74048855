"""Dropout as a torch module over the library's kernel: the mask follows from a counter and is never stored.

    drop = Dropout(0.1)
    y = drop(x)                          # like torch.nn.Dropout(0.1)
    stream = drop(branch, stream)        # stream + dropped branch, in one pass

Every call in training draws anew.  Without a seed its mask is that of a number from torch's generator on the CPU: torch.manual_seed
repeats a run, and a function that is run again for its gradients (torch.utils.checkpoint) has the masks of its first run.  With a seed
the mask is that of the seed and the number of calls before it, which is in the module's state_dict: modules need seeds of their own, and a
function that is run again draws anew.  A captured graph repeats the calls it was captured with; `step`, an int64 tensor on the device that
the program moves between replays, gives each replay masks of its own.  It stays the program's: neither state_dict nor .to() takes it along.
"""
from __future__ import annotations

import torch

from . import binding as nuq
from .draws import Draws, Drawing
from .norm import _rows


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, step):
        x = _rows(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        nuq.nuq_dropout(x, None if residual is None else _rows(residual), p, seed, step, y)
        # (the step's value, not its place: the program may move it before the backward pass)
        ctx.drawn, ctx.step = (p, seed), step.clone() if step is not None else None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dy = _rows(dy)
        dx = None
        if ctx.needs_input_grad[0]:
            dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
            nuq.nuq_dropout(dy, None, *ctx.drawn, ctx.step, dx)
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


class Dropout(Drawing):
    """torch.nn.Dropout with masks of its own; called with a second tensor it adds what is kept to that."""

    def __init__(self, p: float = 0.1, seed: int | None = None, step: torch.Tensor | None = None):
        super().__init__()
        self.draws = Draws(p, seed, step)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None) -> torch.Tensor:
        if x.dim() < 1 or (residual is not None and residual.shape != x.shape):
            raise ValueError("rows are needed, and a residual of the same shape")
        draws = self.draws
        p = draws.p if self.training else 0.0
        if p == 0.0 and residual is None:
            return x
        return _Dropout.apply(x, residual, p, draws.next() if p else 0, draws.step)

    def extra_repr(self) -> str:
        return "p=%g, seed=%s" % (self.draws.p, self.draws.seed)
