"""Modules with a generator of their own inside of torch.utils.checkpoint: the forward pass is computed twice, with the same masks.
On the CPU, with the kernels' calls replaced by their formulas."""
import copy

import pytest
import torch
from torch.utils.checkpoint import checkpoint, set_checkpoint_early_stop

from paper_2306_06098_b200 import dropout as D
from paper_2306_06098_b200 import norm
from philox import kept


def masked(x, p, rng):
    keep = kept(tuple(x.shape), p, *rng.tolist())
    return torch.where(keep, x / (1 - p), torch.zeros_like(x))


def plain_dropout(x, p, rng, residual=None):
    y = masked(x, p, rng)
    return y if residual is None else y + residual


def plain_add_rms_norm(x, residual, weight=None, eps=1e-6, p=0.0, rng=None):
    h = masked(x, p, rng) + residual
    return h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * weight, h


class Block(torch.nn.Module):
    def __init__(self, seed):
        super().__init__()
        self.inner = torch.nn.Linear(16, 16).double()
        self.dropout = D.Dropout(0.5, seed=seed)
        self.norm = norm.RMSNorm(16, p=0.25, seed=seed + 1, dtype=torch.float64)

    def forward(self, x):
        y = torch.tanh(self.inner(self.dropout(x)))
        y, h = self.norm(y, x)
        return self.dropout(torch.sin(y), h)  # (one generator twice)


@pytest.fixture
def on_cpu(monkeypatch):
    monkeypatch.setattr(D, "dropout", plain_dropout)
    monkeypatch.setattr(norm, "add_rms_norm", plain_add_rms_norm)


def blocks():
    torch.manual_seed(1)
    return torch.nn.ModuleList([Block(10), Block(20), Block(30)])


def gradients(model, run, times=1):
    x = torch.linspace(-1, 1, 80, dtype=torch.float64).view(5, 16).requires_grad_(True)
    y = x
    for block in model:
        y = run(block, y)
    leaves = [x, *model.parameters()]
    got = [torch.autograd.grad(y.cos().sum(), leaves, retain_graph=k + 1 < times) for k in range(times)]
    return y.detach(), got


def states(model):
    return [m.rng.tolist() for m in model.modules() if hasattr(m, "rng")]


def with_contexts(block, x):
    return checkpoint(block, x, use_reentrant=False, context_fn=D.checkpoint_contexts)


def nested(block, x):
    return checkpoint(lambda t: with_contexts(block, torch.sin(t)), x, use_reentrant=False, context_fn=D.checkpoint_contexts)


@pytest.mark.parametrize("times", [1, 2])
@pytest.mark.parametrize("run,plain", [(with_contexts, lambda block, x: block(x)), (nested, lambda block, x: block(torch.sin(x)))])
def test_the_masks_are_those_of_the_forward_pass(on_cpu, run, plain, times):
    model = blocks()
    twin = copy.deepcopy(model)
    want, grads = gradients(twin, plain)
    got, all_grads = gradients(model, run, times)
    assert torch.equal(got, want)
    for each in all_grads:
        for a, b in zip(each, grads[0]):
            assert torch.equal(a, b)
    assert states(model) == states(twin)  # moved on once for each call
    again, _ = gradients(model, run)
    assert not torch.equal(again, got)


def test_two_passes_under_way_at_once(on_cpu):
    """Several micro-batches forward before the first goes backward."""
    model = blocks()
    twin = copy.deepcopy(model)
    x = torch.ones(3, 16, dtype=torch.float64, requires_grad=True)

    def go(model, run):
        ys = []
        for _ in range(3):
            y = x
            for block in model:
                y = run(block, y)
            ys.append(y.square().sum())
        return [torch.autograd.grad(y, x)[0] for y in ys]

    for a, b in zip(go(model, with_contexts), go(twin, lambda block, t: block(t))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("reentrant", [False, True])
def test_without_the_contexts_it_is_refused(on_cpu, reentrant):
    """Nothing else would tell that the gradients were another mask's."""
    block = Block(5)
    x = torch.ones(3, 16, dtype=torch.float64, requires_grad=True)
    y = checkpoint(block, x, use_reentrant=reentrant)
    before = states(block)
    with pytest.raises(RuntimeError, match="checkpoint_contexts"):
        y.sum().backward()
    assert states(block) == before
    block.eval()
    checkpoint(torch.nn.Sequential(block.inner, block.dropout), x, use_reentrant=reentrant).sum().backward()


def test_a_pass_that_asks_for_more(on_cpu):
    drop, calls = D.Dropout(0.5, seed=3), []

    def f(x):
        calls.append(0)
        for _ in calls:
            x = torch.sin(drop(x))
        return x

    with set_checkpoint_early_stop(False):
        y = checkpoint(f, torch.ones(8, dtype=torch.float64, requires_grad=True), use_reentrant=False, context_fn=D.checkpoint_contexts)
    with pytest.raises(RuntimeError, match="more generator states"):
        y.sum().backward()
    assert D._tapes() == []


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_on_the_device(dtype):
    torch.manual_seed(2)
    drop, layer = D.Dropout(0.5, seed=7).cuda(), norm.RMSNorm(64, p=0.25, seed=8).cuda()
    twins = copy.deepcopy(drop), copy.deepcopy(layer)

    def f(x, drop, layer):
        y, h = layer(torch.sin(drop(x)), x)
        return drop(y, h)

    x = torch.randn(50, 64, device="cuda").to(dtype).requires_grad_(True)
    grad = torch.randn(50, 64, device="cuda").to(dtype)
    want = torch.autograd.grad(f(x, *twins), (x, twins[1].weight), grad)
    y = checkpoint(f, x, drop, layer, use_reentrant=False, context_fn=D.checkpoint_contexts)
    got = torch.autograd.grad(y, (x, layer.weight), grad)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert drop.rng[1].item() == 2 and layer.rng[1].item() == 1
