"""Dropout, the norm of the residual stream and the linear cross entropy together, as the example that fills in masked
tokens uses them."""
import importlib.util
import os

import pytest
import torch

from philox import kept, threshold

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


def example():
    spec = importlib.util.spec_from_file_location("train_tokens", os.path.join(ROOT, "examples", "train_tokens.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def small(p, seed=3):
    torch.manual_seed(seed)
    mod = example()
    model = mod.Encoder(vocab=77, length=9, d=40, heads=4, layers=2, p=p, seed=seed).cuda()
    with torch.no_grad():  # (ones would hide a weight in the wrong place)
        for m in (model.first, *model.norms):
            m.weight.add_(0.2 * torch.randn_like(m.weight))
    return mod, model, next(mod.batches(5, 9, 77, seed, "cuda"))


def in_64_bits(model, tokens, targets, offset):
    """The loss from elementary operations, with the masks of the generators' `offset`-th use."""
    def drop(x, m):
        p = m.p
        if not p:
            return x
        keep = kept(x.shape, p, int(m.rng[0]), offset).cuda()
        return torch.where(keep, x * (65536 / (65536 - threshold(p))), 0.0)

    def norm(h, m):
        return h / (h.square().mean(-1, keepdim=True) + m.eps).sqrt() * m.weight

    h = drop(model.tokens(tokens) + model.places, model.dropout)
    y = norm(h, model.first)
    for layer, m in zip(model.layers, model.norms):
        h = drop(layer(y).double(), m) + h
        y = norm(h, m)
    used = targets >= 0
    logits = y[used] @ model.tokens.weight.t()
    return (torch.logsumexp(logits, 1) - logits.gather(1, targets[used][:, None])[:, 0]).mean()


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_loss_and_gradients_of_the_whole(p):
    mod, model, (tokens, targets) = small(p)
    params = list(model.parameters())
    loss = model(tokens, targets)
    got = torch.autograd.grad(loss, params)
    twin = mod.Encoder(vocab=77, length=9, d=40, heads=4, layers=2, p=p, seed=3).cuda()
    twin.load_state_dict(model.state_dict())
    twin.double()
    # (softmax in the example's attention is fp32 on both sides: its error is counted as one more rounding)
    want = in_64_bits(twin, tokens, targets, 0)
    grads = torch.autograd.grad(want, list(twin.parameters()))
    # 20 operations one behind the other, sums of up to 160 terms and 8 roundings in each, whose errors a norm or a
    # softmax may scale up by ten
    bound = 20 * (160 + 8) * 10 * U
    assert abs(loss.item() - want.item()) <= bound * abs(want.item())
    for a, b in zip(got, grads):
        assert (a.double() - b).norm() <= bound * b.norm()


def test_captured_in_a_graph():
    _, model, (tokens, targets) = small(0.0)
    params = list(model.parameters())
    loss = model(tokens, targets)
    want, eager = torch.autograd.grad(loss, params), loss.detach()
    del loss  # (torch refuses to capture a backward pass while another graph of the same leaves lives)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(model(tokens, targets), params)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = model(tokens, targets)
        got = torch.autograd.grad(loss, params)
    for _ in range(2):
        for g in got:
            g.zero_()
        graph.replay()
        assert torch.equal(loss, eager)
        for k, (a, b) in enumerate(zip(got, want)):
            # the embedding's own gradient is added up by torch, in any order
            assert torch.equal(a, b) if k else (a - b).abs().max() <= 64 * U * b.abs().max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_example_runs(dtype):
    model, losses = example().train(steps=3, batch=4, length=32, vocab=200, dtype=dtype, log=lambda _: None)
    assert losses.shape == (3,) and losses.isfinite().all()
    assert all(p.isfinite().all() for p in model.parameters())
    assert model.dropout.rng[1].item() == 3 and model.norms[0].rng[1].item() == 3
