"""Numbers for modules that draw: each call of one takes the next."""
from __future__ import annotations

import torch


class Draws:
    """Numbers for calls that draw: from torch's generator, or the seed of a module, moved on by every call."""

    def __init__(self, p: float, seed: int | None, step: torch.Tensor | None):
        if not 0.0 <= p <= 1.0:
            raise ValueError("a probability between 0 and 1")
        self.p, self.seed, self.step, self.calls = p, seed, step, 0

    def next(self) -> int:
        if self.seed is None:
            return int(torch.randint(1 << 62, (), device="cpu"))      # (whatever the default device)
        self.calls += 1
        return (self.seed + self.calls * 0xA0761D6478BD642F) & (1 << 64) - 1     # (odd: no two of 2^64 calls share one)


class Drawing(torch.nn.Module):
    """A module that has `draws`: with a seed the number of calls is part of its state_dict.  (Draws is no module itself: a call takes one
    microsecond longer with an attribute of a module to move.)"""

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        if self.draws.seed is not None:
            destination[prefix + "draws.calls"] = torch.tensor(self.draws.calls, device="cpu")

    def _load_from_state_dict(self, state_dict, prefix, *rest):
        calls = state_dict.pop(prefix + "draws.calls", None)  # (none in a state of a module without a seed: the number stays)
        if calls is not None and self.draws.seed is not None:
            self.draws.calls = int(calls)
        super()._load_from_state_dict(state_dict, prefix, *rest)
