"""Softmax cross entropy of a linear layer in fp32: operands are held as three bfloat16 parts, and six of the parts' nine products are
added up.  Each of them is looked at by itself: operands come in pairs whose other parts cancel, exactly."""
import math

import pytest
import torch

from test_gpu_cross_entropy import B

pytestmark = pytest.mark.gpu

PRODUCTS = ((0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0))


def numbers(count, seed):
    """Values whose parts are about 512, 1 and 2^-9, each with few bits, in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def pick(choices):
        return torch.tensor(choices, dtype=torch.float64, device="cuda")[torch.randint(0, len(choices), (count,), device="cuda", generator=g)]

    return pick([520.0, 640.0, 768.0, 896.0]), pick([1.25, -1.25, 1.5, -1.75]), pick([k * 2.0 ** -14 for k in (40, -40, 24, -56)])


def pair(parts, i):
    """(P, Q) with P - Q the i-th part alone, and all the parts before it in both."""
    return sum(parts[:i + 1]), sum(parts[:i], torch.zeros_like(parts[0]))


def split(x):
    """The bfloat16 parts of fp32 values, in 64 bits."""
    parts, x = [], x.double()
    for _ in range(3):
        parts.append(x.float().to(torch.bfloat16).double())
        x = x - parts[-1]
    return parts


def test_the_parts_are_those():
    parts = numbers(500, 1)
    for i in range(3):
        x, _ = pair(parts, i)
        assert torch.equal(x, x.float().double())
        for k, part in enumerate(split(x)):
            assert torch.equal(part, parts[k] if k <= i else torch.zeros_like(part))


@pytest.mark.parametrize("i,j", PRODUCTS)
def test_logits(i, j):
    n, v = 40, 200
    h, w = numbers(n, 1), numbers(v, 2)
    logits = h[i][:, None] * w[j][None, :]
    scale = 2.0 ** -math.floor(math.log2(logits.abs().max().item()))
    (p, q), (r, s) = pair(h, i), pair(w, j)
    hidden, weight = torch.stack((p, -p, -q, q), 1) * scale, torch.stack((r, s, r, s), 1)
    assert torch.equal(hidden @ weight.t(), logits * scale)
    targets = torch.arange(n, device="cuda")
    losses, lse = B().cross_entropy_forward(hidden.float(), weight.float(), targets, -100, "none")
    want = torch.logsumexp(logits * scale, 1)
    # all sums are exact: what is left are the exponentials of logits of up to 2, and the roundings of results of up to 8
    assert (lse - want).abs().max() <= 2.0 ** -19
    assert (losses - (want - logits.diagonal() * scale)).abs().max() <= 2.0 ** -19
    # without this product all logits would be 0
    assert ((want - math.log(v)).abs() > 2.0 ** -10).all()


def kept(g, x, j, without=None):
    """The j-th part of x times what is kept of g for it."""
    held = [part for k, part in enumerate(split(g)) if (k, j) in PRODUCTS and (k, j) != without]
    return sum(held, torch.zeros_like(g, dtype=torch.float64)).t() @ x


@pytest.mark.parametrize("j", [0, 1, 2])
def test_gradients(j):
    """For either gradient one column holds pairs of rows (of classes, or tokens) that differ there alone, where the other operand is
    0: their entries of the logits' gradient are the same, and the column's gradient is that times the j-th part."""
    n, v, d = 64, 96, 12
    g = torch.Generator(device="cuda").manual_seed(3)
    hidden = torch.randn(n // 2, d, device="cuda", generator=g).repeat_interleave(2, 0)
    weight = torch.randn(v // 2, d, device="cuda", generator=g).repeat_interleave(2, 0)
    hidden[:, :2] = weight[:, :2] = 0
    parts_h, parts_w = numbers(n // 2, 4), numbers(v // 2, 5)
    for to, col, parts in ((hidden, 0, parts_h), (weight, 1, parts_w)):
        p, q = pair(parts, j)
        to[::2, col], to[1::2, col] = p.float(), -q.float()
    grad = (torch.rand(n // 2, device="cuda", generator=g) + 0.5).repeat_interleave(2)
    targets = torch.full((n,), v - 3, device="cuda")  # (of no pair that is looked at: both halves of it have other entries)
    weight[v - 4:, 1] = 0
    parts_w[j][-2:] = 0
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dh, dw = B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none")
    G = torch.softmax(hidden.double() @ weight.double().t(), 1)
    G[:, v - 3] -= 1
    G = (grad.double()[:, None] * G)
    left = 12 * 2.0 ** -24 if j == 0 else 2.0 ** -15 if j == 1 else 2.0 ** -7  # G's own error; what the products that are left out hold of it
    for got, each, part in ((dh[:, 1], G[:, ::2].t(), parts_w[j]), (dw[:-4, 0], G[::2, :-4], parts_h[j])):
        want = each.t() @ part
        assert (got.double() - want).norm() <= left * want.norm()
        # a product more left out
        for k in range(3 - j):
            lost = kept(each.float(), part, j, (k, j))
            assert (lost - want).norm() > left * want.norm()
        assert (kept(each.float(), part, j) - want).norm() <= left * want.norm()


@pytest.mark.parametrize("n,d,v", [(1003, 509, 10007), (300, 72, 513), (2500, 96, 5003)])
def test_as_exact_as_fp32(n, d, v):
    """The errors' 2-norm on ordinary inputs: a few roundings of fp32.  With three products instead of six it is 7e-7 and more."""
    from test_gpu_cross_entropy import inputs
    hidden, weight, targets = inputs(n, d, v, torch.float32, 1)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dh, dw = B().cross_entropy_backward(torch.ones((), device="cuda"), hidden, weight, targets, lse, -100, "sum")
    h, w = hidden.double(), weight.double()
    G = torch.softmax(h @ w.t(), 1)
    G[torch.arange(n), targets] -= 1
    for got, want in ((dh, G @ w), (dw, G.t() @ h)):
        assert (got - want).norm() <= 8 * 2.0 ** -24 * want.norm()
    (a, b), (c, e) = (split(t)[:2] for t in (h, w))
    three = torch.softmax(a @ c.t() + a @ e.t() + b @ c.t(), 1)
    three[torch.arange(n), targets] -= 1
    assert (three @ w - G @ w).norm() > 8 * 2.0 ** -24 * (G @ w).norm()
