"""Norms as torch modules over the library's kernels, with the sum of a residual stream taken on the way.

    norm = LayerNorm(1600)
    y = norm(x)                          # like torch.nn.LayerNorm(1600)
    y, stream = norm(branch, stream)     # stream + branch, and its norm: between two blocks of a transformer

    seam = ResidualNorm(1600, inner="rms", outer="rms", gate=0.1, dropout=0.1)
    y, stream = seam(branch, stream)     # the same with a norm of the branch, a gate per column, dropout and scales before the sum

Rows in float32, bfloat16 or float16; weight and bias in the rows' type or in float32.  Nothing here computes: the forward and
the backward pass are one call of the library each.
"""
from __future__ import annotations

import torch

from . import binding as nuq
from .draws import Draws, Drawing


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy of it whose rows the kernels take."""
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        return t
    return t.contiguous() if t.numel() else t.new_empty(t.shape)         # (no elements are contiguous whatever their strides)


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
    """torch.nn.LayerNorm over the last dimension; called with a second tensor it norms the sum and returns that too.  (ResidualNorm: the
    same with other norms, a norm of the branch, a gate, dropout and scales.)"""

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


_KINDS = {None: nuq.NO_NORM, "layer": nuq.LAYER_NORM, "rms": nuq.RMS_NORM}


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, w1, b1, gate, w2, b2, inner, outer, eps, scale, residual_scale, p, seed, step):
        x = _rows(x)
        rows = x.numel() // x.shape[-1]
        total = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        y = torch.empty_like(total) if outer != nuq.NO_NORM else None
        stats = torch.empty(4, rows, dtype=torch.float32, device=x.device)
        nuq.nuq_residual_norm_forward(x, None if residual is None else _rows(residual), inner, w1, b1, gate, outer, w2, b2, eps, scale,
                                      residual_scale, p, seed, step, total, y, stats)
        # (the step's value, not its place: the program may move it before the backward pass)
        ctx.save_for_backward(x, total if y is not None else None, w1, b1, gate, w2, b2, stats, step.clone() if step is not None else None)
        ctx.numbers = (inner, outer, scale, residual_scale, p, seed)
        ctx.set_materialize_grads(False)
        return total if y is None else (y, total)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        x, total, w1, b1, gate, w2, b2, stats, step = ctx.saved_tensors
        inner, outer, scale, residual_scale, p, seed = ctx.numbers
        dy, dtotal = grads if outer != nuq.NO_NORM else (None, grads[0])
        if dy is None and dtotal is None:
            return (None,) * 15
        factor = w2
        if dy is None and outer != nuq.NO_NORM:              # the norm itself was not used: as of a norm of rows of 0, whatever total holds
            dy = total = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
            stats, factor = torch.cat([stats[:2], torch.zeros_like(stats[2:])]), None
        need = ctx.needs_input_grad
        empty = lambda v, k: torch.empty_like(v) if v is not None and need[k] else None  # noqa: E731
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dresidual = torch.empty_like(dx) if need[1] else None
        dw1, db1, dgate, dw2, db2 = (empty(v, k) for v, k in zip((w1, b1, gate, w2, b2), range(2, 7)))
        workspace = None
        if any(v is not None for v in (dw1, db1, dgate, dw2, db2)):
            workspace = torch.empty(nuq.nuq_residual_norm_workspace_bytes(stats.shape[1], x.shape[-1]), dtype=torch.uint8, device=x.device)
        nuq.nuq_residual_norm_backward(None if dy is None else _rows(dy), None if dtotal is None else _rows(dtotal), x,
                                       total, inner, w1, b1, gate, outer, factor, scale, residual_scale, p,
                                       seed, step, stats, dx, dresidual, dw1, db1, dgate, dw2, db2, workspace)
        return (dx, dresidual, dw1, db1, dgate, dw2, db2) + (None,) * 8


class ResidualNorm(Drawing):
    """The seam between two blocks: `inner` norms the branch, `outer` the sum ("layer", "rms", or None; one of them at least).

    seam(branch, stream) is (y, stream') with stream' = residual_scale stream + scale drop(gate norm(branch)) and y its norm, or stream'
    alone without an outer norm.  gate: the value its weights begin with, or None for no gate.  Dropout draws as dropout.Dropout does.
    A layer norm of the plain sum is LayerNorm(branch, stream), whose backward pass writes one gradient for both."""

    def __init__(self, hidden: int, inner: str | None = None, outer: str | None = "layer", gate: float | None = None, scale: float = 1.0,
                 residual_scale: float = 1.0, dropout: float = 0.0, eps: float = 1e-5, bias: bool = True, seed: int | None = None,
                 step: torch.Tensor | None = None, device=None, dtype=None):
        super().__init__()
        if not 1 <= hidden <= nuq.RESIDUAL_NORM_MAX_HIDDEN:
            raise ValueError("rows of 1 to %d elements" % nuq.RESIDUAL_NORM_MAX_HIDDEN)
        if inner not in _KINDS or outer not in _KINDS or (inner is None and outer is None):
            raise ValueError("norms are \"layer\", \"rms\" or None, and not both None")
        self.hidden, self.inner, self.outer, self.eps = hidden, inner, outer, eps
        self.scale, self.residual_scale, self.draws = scale, residual_scale, Draws(dropout, seed, step)
        vector = lambda value: torch.nn.Parameter(torch.full((hidden,), value, device=device, dtype=dtype))  # noqa: E731
        self.inner_weight = vector(1.0) if inner else None
        self.inner_bias = vector(0.0) if inner and bias else None
        self.gate = vector(gate) if gate is not None else None
        self.outer_weight = vector(1.0) if outer else None
        self.outer_bias = vector(0.0) if outer and bias else None

    def forward(self, branch: torch.Tensor, stream: torch.Tensor | None = None):
        if branch.shape[-1:] != (self.hidden,) or (stream is not None and stream.shape != branch.shape):
            raise ValueError("rows of %d are needed, and a stream of the same shape" % self.hidden)
        draws = self.draws
        p = draws.p if self.training else 0.0
        return _ResidualNorm.apply(branch, stream, self.inner_weight, self.inner_bias, self.gate, self.outer_weight, self.outer_bias,
                                   _KINDS[self.inner], _KINDS[self.outer], self.eps, self.scale, self.residual_scale, p,
                                   draws.next() if p else 0, draws.step)

    def extra_repr(self) -> str:
        return "%d, inner=%s, outer=%s, gate=%s, scale=%g, residual_scale=%g, dropout=%g, eps=%g" % (
            self.hidden, self.inner, self.outer, self.gate is not None, self.scale, self.residual_scale, self.draws.p, self.eps)
