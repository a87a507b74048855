"""Softmax cross entropy of a language model over the library's kernels: the read-out product and the loss in one, without the logits.

    loss = linear_cross_entropy(x, weight, target)           # like cross_entropy(x @ weight.t(), target), [rows, vocab] never in memory
    head = LinearCrossEntropy(1600, 50257)                   # the same with the weights as a parameter
    loss = head(x, target)

x [..., hidden] and weight [vocabulary, hidden] in float32, bfloat16 or float16, target [...] int64.  A weight of another type than x's
is cast to it on the way, its gradient back: beside rows in 16 bits a weight in float32 has a gradient that was rounded to 16 bits.  A target
outside the vocabulary makes its row's loss NaN, with a gradient of 0, and raises FLAG_MALFORMED (nuq_last_error_flags).
"""
from __future__ import annotations

import math

import torch

from . import binding as nuq
from .norm import _rows


def _workspace(x, weight, backward):
    return torch.empty(nuq.nuq_linear_cross_entropy_workspace_bytes(x, weight, backward), dtype=torch.uint8, device=x.device)


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target, ignore, smoothing, mean):
        x, weight, target = _rows(x), _rows(weight), target.contiguous()
        loss = torch.empty(target.shape, dtype=torch.float32, device=x.device)
        lse = torch.empty(target.numel(), dtype=torch.float32, device=x.device)
        both = torch.empty(2, dtype=torch.float32, device=x.device) if mean else None
        nuq.nuq_linear_cross_entropy_forward(x, weight, target, ignore, smoothing, loss, lse, both, _workspace(x, weight, False))
        ctx.save_for_backward(x, weight, target, lse, both)
        ctx.numbers = (ignore, smoothing)
        # (not a view, which autograd would not let the program change in place; the backward pass reads both[1] alone)
        return both[0].data if mean else loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, target, lse, both = ctx.saved_tensors
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if ctx.needs_input_grad[0] else None
        dweight = torch.empty(weight.shape, dtype=weight.dtype, device=weight.device) if ctx.needs_input_grad[1] else None
        if lse.numel() == 1 and both is None:                # (one row: its gradient is the one number)
            grad = grad.reshape(1)
        nuq.nuq_linear_cross_entropy_backward(x, weight, target, *ctx.numbers, lse, grad.contiguous(), both, dx, dweight,
                                              _workspace(x, weight, True))
        return dx, dweight, None, None, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, ignore: int = -100, smoothing: float = 0.0,
                         reduction: str = "mean") -> torch.Tensor:
    """The mean loss over the rows whose target is not `ignore` (0 where there are none), or with reduction "none" every row's."""
    if reduction not in ("mean", "none"):
        raise ValueError("reduction: \"mean\" or \"none\"")
    if x.dim() < 1 or weight.dim() != 2 or weight.shape[1:] != x.shape[-1:] or target.shape != x.shape[:-1]:
        raise ValueError("x [..., hidden], weight [vocabulary, hidden] and target [...] are needed")
    if target.dtype is not torch.int64:
        raise ValueError("target: int64 is needed")
    return _LinearCrossEntropy.apply(x, weight.to(x.dtype), target, ignore, smoothing, reduction == "mean")


class LinearCrossEntropy(torch.nn.Module):
    """The read-out of a language model and its loss: weight [vocab, hidden], without a bias."""

    def __init__(self, hidden: int, vocab: int, ignore: int = -100, smoothing: float = 0.0, device=None, dtype=None):
        super().__init__()
        if hidden < 1 or vocab < 1 or not 0.0 <= smoothing < 1.0:
            raise ValueError("a width, a vocabulary and a smoothing below 1")
        self.ignore, self.smoothing = ignore, smoothing
        self.weight = torch.nn.Parameter(torch.randn(vocab, hidden, device=device, dtype=dtype) / math.sqrt(hidden))

    def forward(self, x: torch.Tensor, target: torch.Tensor, reduction: str = "mean") -> torch.Tensor:
        return linear_cross_entropy(x, self.weight, target, self.ignore, self.smoothing, reduction)

    def extra_repr(self) -> str:
        return "%d, vocab=%d, ignore=%d, smoothing=%g" % (self.weight.shape[1], self.weight.shape[0], self.ignore, self.smoothing)
