"""Layer norm as a torch module over the library's kernels, with the sum of a residual stream taken on the way.

    norm = LayerNorm(1600)
    y = norm(x)                          # like torch.nn.LayerNorm(1600)
    y, stream = norm(branch, stream)     # stream + branch, and its norm: between two blocks of a transformer

Rows in float32, bfloat16 or float16; weight and bias in the rows' type or in float32.  Nothing here computes: the forward and
the backward pass are one call of the library each.
"""
from __future__ import annotations

import torch

from . import binding as nuq


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy of it whose rows the kernels take."""
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        return t
    return t.contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps):
        x = _rows(x)
        rows = x.numel() // x.shape[-1]
        total = torch.empty(x.shape, dtype=x.dtype, device=x.device) if residual is not None else None
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty(2, rows, dtype=torch.float32, device=x.device)
        nuq.nuq_layer_norm_forward(x, None if residual is None else _rows(residual), weight, bias, eps, total, y, stats[0], stats[1])
        ctx.save_for_backward(x if total is None else total, weight, bias, stats)
        ctx.set_materialize_grads(False)
        return y if total is None else (y, total)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dtotal=None):
        s, weight, bias, stats = ctx.saved_tensors
        if dy is None:                       # the norm itself was not used
            return dtotal, dtotal, None, None, None
        rows, hidden = stats.shape[1], s.shape[-1]
        dx = torch.empty(s.shape, dtype=s.dtype, device=s.device)
        dweight = torch.empty_like(weight) if weight is not None and ctx.needs_input_grad[2] else None
        dbias = torch.empty_like(bias) if bias is not None and ctx.needs_input_grad[3] else None
        workspace = None
        if dweight is not None or dbias is not None:
            workspace = torch.empty(nuq.nuq_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=s.device)
        nuq.nuq_layer_norm_backward(_rows(dy), s, weight, stats[0], stats[1], None if dtotal is None else _rows(dtotal), dx,
                                    dweight, dbias, workspace)
        return dx, dx if ctx.needs_input_grad[1] else None, dweight, dbias, None


class LayerNorm(torch.nn.Module):
    """torch.nn.LayerNorm over the last dimension; called with a second tensor it norms the sum and returns that too."""

    def __init__(self, hidden: int, eps: float = 1e-5, elementwise_affine: bool = True, bias: bool = True, device=None, dtype=None):
        super().__init__()
        if hidden < 1:
            raise ValueError("rows of one element or more")
        self.hidden, self.eps = hidden, eps
        new = dict(device=device, dtype=dtype)
        self.weight = torch.nn.Parameter(torch.ones(hidden, **new)) if elementwise_affine else None
        self.bias = torch.nn.Parameter(torch.zeros(hidden, **new)) if elementwise_affine and bias else None

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        if x.shape[-1:] != (self.hidden,) or (residual is not None and residual.shape != x.shape):
            raise ValueError("rows of %d are needed, and a residual of the same shape" % self.hidden)
        return _LayerNorm.apply(x, residual, self.weight, self.bias, self.eps)

    def extra_repr(self) -> str:
        return "%d, eps=%g, affine=%s, bias=%s" % (self.hidden, self.eps, self.weight is not None, self.bias is not None)
