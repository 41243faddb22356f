"""Group normalisation for training with torch.autograd (argument marshalling only): both
directions run in the CUDA library behind `binding`.

Group normalisation takes the statistics of each sample by itself: samples of a batch do not depend on each
other, and results not on the batch size.  The optimizer works with any model; this is one that a model may use.
"""
from typing import Optional

import torch

from . import binding


class _GroupNormAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act):
        y, mean, rstd = binding.group_norm_forward(x, groups, weight, bias, eps, act)
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        ctx.groups, ctx.act = groups, act
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, mean, rstd, weight, bias = ctx.saved_tensors
        dx, dweight, dbias = binding.group_norm_backward(dy, x, mean, rstd, ctx.groups, weight,
                                                         bias, ctx.act)
        return dx, dweight, dbias, None, None, None


def group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               act: str = "none") -> torch.Tensor:
    """act(group_norm(x)) with gradients; x (n, channels, *positions), channels last in memory
    (other layouts are copied).  act: "none", "relu" or "silu"."""
    return _GroupNormAct.apply(x, weight, bias, groups, eps, act)


class GroupNorm(torch.nn.Module):
    """torch.nn.GroupNorm(groups, channels) followed by `act`, in one pass and channels last."""

    def __init__(self, groups: int, channels: int, eps: float = 1e-5, affine: bool = True,
                 act: str = "none", device=None, dtype=None):
        super().__init__()
        if groups < 1 or channels < 1 or channels % groups:
            raise ValueError("channels must be a positive multiple of groups")
        if act not in binding.ACTS:
            raise ValueError(f"act: one of {', '.join(binding.ACTS)} expected, got {act!r}")
        self.groups, self.channels, self.eps, self.act = groups, channels, eps, act
        if affine:
            self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))
            self.bias = torch.nn.Parameter(torch.zeros(channels, device=device, dtype=dtype))
        else:
            self.register_parameter("weight", None)
            self.register_parameter("bias", None)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return group_norm(x, self.groups, self.weight, self.bias, self.eps, self.act)

    def extra_repr(self) -> str:
        return (f"{self.groups}, {self.channels}, eps={self.eps}, "
                f"affine={self.weight is not None}, act={self.act}")
