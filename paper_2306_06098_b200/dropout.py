"""Dropout for training with torch.autograd (argument marshalling only): the CUDA library behind `binding`
computes the mask from a counter in both directions, and nothing but the counter is kept in between.
"""
import threading
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
        saved = ctx.saved_tensors  # (a checkpointed pass hands them out once)
        rng = saved[0] if saved else ctx.rng
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
    each replay.  Where torch.utils.checkpoint computes a forward pass again, inside the backward pass, the masks
    have to be those of the first time: see `checkpoint_contexts`, without which this raises there."""
    tapes = _tapes()
    again = max((i for i, t in enumerate(tapes) if t.again), default=-1)
    if again >= 0:
        now = tapes[again].next()
    elif torch._C._current_graph_task_id() != -1:
        raise RuntimeError("a generator was asked for its next state inside a backward pass, where it would give another mask "
                           "than in the forward pass: use torch.utils.checkpoint.checkpoint(..., use_reentrant=False, "
                           "context_fn=dropout.checkpoint_contexts)")
    else:
        now = rng.clone()
        rng[1:].add_(1)
    for t in tapes[again + 1:]:
        t.states.append(now)
    return now


_local = threading.local()  # (a backward pass has threads of its own)


def _tapes() -> list:
    if not hasattr(_local, "tapes"):
        _local.tapes = []
    return _local.tapes


class _Tape:
    """Inside of it states that are taken are written down, or (again) come from what was written."""

    def __init__(self, states: list, again: bool):
        self.states, self.again, self.at = states, again, 0

    def next(self) -> torch.Tensor:
        if self.at == len(self.states):
            raise RuntimeError("a forward pass that was computed again asked for more generator states than the first time")
        self.at += 1
        return self.states[self.at - 1]

    def __enter__(self):
        self.at = 0
        _tapes().append(self)

    def __exit__(self, *_):
        _tapes().remove(self)


def checkpoint_contexts():
    """The context_fn for torch.utils.checkpoint.checkpoint(f, ..., use_reentrant=False): modules with a generator of
    their own take the same states, and so draw the same masks, when f is computed again."""
    states = []
    return _Tape(states, False), _Tape(states, True)


class WithGenerator(torch.nn.Module):
    """A module with a generator of its own: its state `rng` (None: it has none) is saved, loaded and moved with the module.
    It is no buffer, since DistributedDataParallel gives all processes the buffers of the first one before each forward
    pass: they would drop the same elements of their own batches.  (They do when they are given equal seeds.)"""
    rng: Optional[torch.Tensor] = None

    def _apply(self, fn, *args, **kwargs):
        super()._apply(fn, *args, **kwargs)
        if self.rng is not None:
            self.rng = fn(self.rng)
        return self

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        if self.rng is not None:
            destination[prefix + "rng"] = self.rng

    def _load_from_state_dict(self, state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys,
                              error_msgs):
        super()._load_from_state_dict(state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys,
                                      error_msgs)
        name = prefix + "rng"
        if self.rng is None:
            return
        if name not in state_dict:
            if strict:
                missing_keys.append(name)
            return
        if name in unexpected_keys:
            unexpected_keys.remove(name)
        given = state_dict[name]
        if not isinstance(given, torch.Tensor) or given.shape != self.rng.shape or given.dtype != self.rng.dtype:
            error_msgs.append(f"{name}: an int64 tensor of (seed, offset) expected")
        elif local_metadata.get("assign_to_params_buffers", False):
            self.rng = given
        else:
            self.rng.copy_(given)


class Dropout(WithGenerator):
    """torch.nn.Dropout(p) with a generator of its own (saved with the model, so that it goes on with the same masks);
    forward(x, residual) adds the residual in the same pass.  Inside of torch.utils.checkpoint: see
    `checkpoint_contexts`."""

    def __init__(self, p: float = 0.5, seed: Optional[int] = None, device=None):
        super().__init__()
        if not 0 <= p <= 1:
            raise ValueError("p: between 0 and 1")
        self.p = p
        self.rng = new_rng(seed, device)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if not self.training or self.p == 0:
            return x if residual is None else x + residual
        return dropout(x, self.p, take(self.rng), residual)

    def extra_repr(self) -> str:
        return f"p={self.p}"
