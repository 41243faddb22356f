"""Softmax cross entropy of a linear layer over a large vocabulary, for training with torch.autograd (argument
marshalling only): the CUDA library behind `binding` never keeps the logits, in either direction.
"""
import torch

from . import binding


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, ignore_index, reduction):
        losses, lse = binding.cross_entropy_forward(hidden, weight, targets, ignore_index, reduction)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.how = ignore_index, reduction
        return losses

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        dhidden, dweight = binding.cross_entropy_backward(grad, *ctx.saved_tensors, *ctx.how,
                                                          ctx.needs_input_grad[:2])
        return dhidden, dweight, None, None, None


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                         ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """torch.nn.functional.cross_entropy(hidden @ weight.t(), targets) in fp32, with gradients of hidden
    (..., d) and weight (vocabulary, d), which have one type.  Tokens whose target is ignore_index cost
    nothing; with reduction "mean" and none left the result is NaN, as there."""
    return _LinearCrossEntropy.apply(hidden, weight, targets, ignore_index, reduction)


class LinearCrossEntropy(torch.nn.Module):
    """A linear layer without bias and its cross entropy: forward(hidden, targets) is the loss.  The weight
    (classes, d) may be another module's, an embedding's for instance; it is used in hidden's type."""

    def __init__(self, d: int, classes: int, weight: torch.nn.Parameter = None, ignore_index: int = -100,
                 reduction: str = "mean", device=None, dtype=None):
        super().__init__()
        if reduction not in ("none", "mean", "sum"):
            raise ValueError(f"reduction: one of none, mean, sum expected, got {reduction!r}")
        if weight is None:
            if d < 1 or classes < 1:
                raise ValueError("d and classes must be positive")
            weight = torch.nn.Parameter(torch.empty(classes, d, device=device, dtype=dtype))
            torch.nn.init.normal_(weight, std=d ** -0.5)
        elif tuple(weight.shape) != (classes, d):
            raise ValueError(f"weight: ({classes}, {d}) expected, got {tuple(weight.shape)}")
        self.weight, self.ignore_index, self.reduction = weight, ignore_index, reduction

    def forward(self, hidden: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        return linear_cross_entropy(hidden, self.weight.to(hidden.dtype), targets, self.ignore_index,
                                    self.reduction)

    def extra_repr(self) -> str:
        classes, d = self.weight.shape
        return f"{d}, {classes}, ignore_index={self.ignore_index}, reduction={self.reduction}"
