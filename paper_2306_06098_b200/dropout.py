"""Dropout for training with torch.autograd (argument marshalling only): the CUDA library behind `binding`
computes the mask from a counter in both directions, and nothing but the counter is kept in between.
"""
from typing import Optional

import torch

from . import binding


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, rng):
        ctx.p, ctx.rng = p, None if isinstance(rng, torch.Tensor) else rng
        ctx.save_for_backward(*(() if ctx.rng is not None or rng is None else (rng,)))
        ctx.residual = residual is not None
        return binding.dropout(x, p, rng, residual)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        rng = ctx.saved_tensors[0] if ctx.saved_tensors else ctx.rng
        dx = binding.dropout(dy, ctx.p, rng) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.residual else None, None, None


def dropout(x: torch.Tensor, p: float, rng, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A share p of x zeroed and the rest scaled by 1 / (1 - p) (p to the nearest 1 / 65536), plus
    `residual`, with gradients.  rng: (seed, offset), ints or an int64 tensor of two on x's device; equal ones give
    equal masks, and a tensor must not change between the two directions (see `take`)."""
    return _Dropout.apply(x, residual, p, rng)


def new_rng(seed: Optional[int] = None, device=None) -> torch.Tensor:
    """A generator's state, (seed, 0); the seed comes from torch's own generator when none is given."""
    if seed is None:
        seed = int(torch.randint(-2 ** 63, 2 ** 63 - 1, (1,)))
    seed = (int(seed) + 2 ** 63) % 2 ** 64 - 2 ** 63
    return torch.tensor([seed, 0], dtype=torch.int64, device=device)


def take(rng: torch.Tensor) -> torch.Tensor:
    """The state to use now, as a copy; `rng` moves on to the next one, on the device: in a captured graph at
    each replay."""
    now = rng.clone()
    rng[1:].add_(1)
    return now


class Dropout(torch.nn.Module):
    """torch.nn.Dropout(p) with a generator of its own, in a buffer (so that a checkpoint goes on with the
    same masks); forward(x, residual) adds the residual in the same pass."""

    def __init__(self, p: float = 0.5, seed: Optional[int] = None, device=None):
        super().__init__()
        if not 0 <= p <= 1:
            raise ValueError("p: between 0 and 1")
        self.p = p
        self.register_buffer("rng", new_rng(seed, device))

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if not self.training or self.p == 0:
            return x if residual is None else x + residual
        return dropout(x, self.p, take(self.rng), residual)

    def extra_repr(self) -> str:
        return f"p={self.p}"
