"""Group normalisation, and root-mean-square normalisation of a residual stream, for training with
torch.autograd (argument marshalling only): both directions run in the CUDA library behind `binding`.

Group normalisation takes the statistics of each sample by itself: samples of a batch do not depend on each
other, and results not on the batch size.  The optimizer works with any model; this is one that a model may use.
"""
from typing import Optional, Tuple

import torch

from . import binding
from .dropout import WithGenerator, new_rng, take


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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, p, rng):
        y, h, rstd = binding.rms_norm_forward(x, weight, eps, residual, p, rng)
        ctx.p, ctx.rng = p, None if isinstance(rng, torch.Tensor) else rng
        ctx.save_for_backward(h, rstd, weight, rng if isinstance(rng, torch.Tensor) else None)
        ctx.set_materialize_grads(False)
        if residual is None and p == 0:
            return y
        return y, h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        h, rstd, weight, rng = ctx.saved_tensors
        if dy is None and dh is None:
            return (None,) * 6
        if dy is None:
            dy = torch.zeros_like(h, memory_format=torch.contiguous_format)
        dx, dresidual, dweight = binding.rms_norm_backward(
            dy, h, rstd, weight, dh, ctx.p, ctx.rng if rng is None else rng, ctx.needs_input_grad[:3])
        return dx, dresidual, dweight, None, None, None


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6) -> torch.Tensor:
    """x / sqrt(mean(x^2) + eps) * weight over the last dimension, with gradients."""
    return _RmsNorm.apply(x, None, weight, eps, 0.0, None)


def add_rms_norm(x: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, p: float = 0.0, rng=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(rms_norm(h), h) of h = dropout(x) + residual in one pass, with gradients; rng as in
    dropout.dropout."""
    return _RmsNorm.apply(x, residual, weight, eps, p, rng)


class RMSNorm(WithGenerator):
    """Root-mean-square norm of the last dimension, of size d.  forward(x) normalises x, and drops nothing;
    forward(x, residual) returns the norm of h = dropout(x) + residual, and h.  The dropout of share p is
    active in training, with a generator of its own (inside of torch.utils.checkpoint: see
    dropout.checkpoint_contexts)."""

    def __init__(self, d: int, eps: float = 1e-6, affine: bool = True, p: float = 0.0,
                 seed: Optional[int] = None, device=None, dtype=None):
        super().__init__()
        if d < 1:
            raise ValueError("d must be positive")
        if not 0 <= p <= 1:
            raise ValueError("p: between 0 and 1")
        self.d, self.eps, self.p = d, eps, p
        self.rng = new_rng(seed, device) if p else None
        if affine:
            self.weight = torch.nn.Parameter(torch.ones(d, device=device, dtype=dtype))
        else:
            self.register_parameter("weight", None)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None):
        if x.shape[-1] != self.d:
            raise ValueError(f"x: {self.d} columns expected, got {x.shape[-1]}")
        if residual is None:
            return rms_norm(x, self.weight, self.eps)
        if not self.training or not self.p:
            return add_rms_norm(x, residual, self.weight, self.eps)
        return add_rms_norm(x, residual, self.weight, self.eps, self.p, take(self.rng))

    def extra_repr(self) -> str:
        return f"{self.d}, eps={self.eps}, affine={self.weight is not None}, p={self.p}"
