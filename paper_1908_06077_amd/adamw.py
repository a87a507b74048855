"""Alg. 1 with AdamW as the parameter update: K coded gradients are averaged, their norm is clipped, and the weights move.

Buffer management around the library calls only, as in sgd.py: encode and decode as there (the decoder writes the average),
then nuq_gradient_norm where gradients are clipped, and one AdamW step on all tensors, its moments in 32 bits or in 8.
"""
from __future__ import annotations

import torch

from . import binding as nuq
from .sgd import DataParallelSGD


class Moments:
    """The two moments of tensors that stand at `starts` in a flat vector of d elements, zero at first.

    bits = 32: fp32.  bits = 8: codes, with two scales per block of nuq.STATE_BLOCK elements; every start is a multiple of it."""

    def __init__(self, sizes: list[int], starts: list[int], d: int, bits: int, device: torch.device):
        if bits not in (8, 32):
            raise ValueError("states of 8 or 32 bits")
        self.bits = bits
        if bits == 32:
            self.flat = {"m": torch.zeros(d, dtype=torch.float32, device=device),
                         "v": torch.zeros(d, dtype=torch.float32, device=device)}
        else:
            if any(o % nuq.STATE_BLOCK for o in starts):
                raise ValueError("a tensor begins inside a block of states")
            self.flat = {"m": torch.zeros(d, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                         "v": torch.zeros(d, dtype=torch.uint8, device=device),
                         "scales": torch.zeros(2 * nuq.nuq_state_blocks(d), dtype=torch.float32, device=device)}
            blocks = [(2 * (o // nuq.STATE_BLOCK), 2 * nuq.nuq_state_blocks(n)) for n, o in zip(sizes, starts)]
            self.scales = [self.flat["scales"][b:b + k] for b, k in blocks]
        self.m, self.v = ([self.flat[x][o:o + n] for n, o in zip(sizes, starts)] for x in ("m", "v"))

    def step(self, which: list[int], ws, grads, decays, alpha, beta1, beta2, eps, t, coefficient=None) -> None:
        pick = lambda xs: [xs[i] for i in which]  # noqa: E731
        hyper = (decays, alpha, beta1, beta2, eps, t, coefficient)
        if self.bits == 32:
            nuq.nuq_adamw_step(ws, grads, pick(self.m), pick(self.v), *hyper)
        else:
            nuq.nuq_adamw_step_coded(ws, grads, pick(self.m), pick(self.v), pick(self.scales), *hyper)


class DataParallelAdamW(DataParallelSGD):
    """Alg. 1's loop on a flat fp32 parameter vector w whose tensors, of `sizes` elements, stand at `starts`; gaps stay zero.

    groups: the hyper-parameters, read at every step: dicts with "which" (indexes of tensors), "lr", "betas", "eps" and
    "weight_decay".  max_norm: the averaged gradient is scaled down to that norm."""

    def __init__(self, w: torch.Tensor, sizes: list[int], starts: list[int], groups: list[dict], K: int, bucket: int, s: int,
                 sync_stride: int = 256, max_norm: float | None = None, state_bits: int = 32, seed: int = 0):
        super().__init__(w, K, 0.0, bucket, s, sync_stride=sync_stride, seed=seed)
        if max_norm is not None and not max_norm > 0.0:
            raise ValueError("a positive norm to clip to")
        if any(o < 0 or o + n > self.d for n, o in zip(sizes, starts)):
            raise ValueError("tensors inside the flat vector")
        self.groups, self.max_norm = groups, max_norm
        self.moments = Moments(sizes, starts, self.d, state_bits, w.device)
        self.average = torch.empty_like(w)
        views = lambda flat: [flat[o:o + n] for n, o in zip(sizes, starts)]  # noqa: E731
        self.ws, self.grads = views(w), views(self.average)
        # norm of the last average, factor on it; NaN before the first step, and where nothing is clipped
        self.norm = torch.full((2,), float("nan"), dtype=torch.float32, device=w.device)
        self.workspace = torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=w.device)

    def apply(self, messages: list[nuq.Message]) -> None:
        """Receiver half: DECODE and average the K messages, clip, move w."""
        nuq.nuq_decode_accumulate(messages, self.d, self.bucket, self.s, self.sync_stride, 1.0 / self.K, False, self.average)
        coefficient = None
        if self.max_norm is not None:
            nuq.nuq_gradient_norm([self.average], self.max_norm, self.workspace, self.norm)
            coefficient = self.norm[1:]
        self.t += 1
        calls: dict[tuple, tuple[list, list]] = {}           # one per set of numbers: groups often differ in their decay alone
        for g in self.groups:
            which, decays = calls.setdefault((g["lr"], *g["betas"], g["eps"]), ([], []))
            which += g["which"]
            decays += [g["weight_decay"]] * len(g["which"])
        for (lr, beta1, beta2, eps), (which, decays) in calls.items():
            self.moments.step(which, [self.ws[i] for i in which], [self.grads[i] for i in which], decays, lr, beta1, beta2, eps,
                              self.t, coefficient)
