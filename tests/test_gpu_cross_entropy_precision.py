"""Softmax cross entropy of a linear layer: what its roundings leave, held to bounds that a mistake in one part alone exceeds.
Such mistakes are planted in the 64-bit results, which then have to lie outside of the bounds."""
import math

import pytest
import torch

from test_gpu_cross_entropy import HALF, SUM, TINY, U, B, definition, grads, inputs

pytestmark = pytest.mark.gpu


def inside(got, want, bound, dtype):
    return ((got.double() - want).abs() <= bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype]).all()


# few tokens next to the classes, so that the targets' entries make up the gradients; d that is no multiple of a tile; one tile of
# classes; several pieces of the vocabulary, as they are and widened
@pytest.mark.parametrize("n,d,v,labelled", [(40, 64, 3000, 1.0), (300, 72, 5003, 1.0), (130, 300, 4096, 0.5), (14, 40, 120, 1.0),
                                            (16300, 24, 30011, 1.0), (16300, 24, 30011, 0.1), (16300, 40, 9001, 0.01), (2500, 128, 30522, 1.0), (40, 8, 300000, 1.0),
                                            (200, 520, 60000, 1.0), (12, 24, 100000, 1.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_entries_of_the_targets(n, d, v, labelled, dtype):
    """Both gradients, where the other entries of the logits' gradient are rounded to the operands' type once, and those of the
    targets are not."""
    hidden, weight, targets = inputs(n, d, v, dtype, 7, labelled, size=0.05)
    grad = grads(n)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dh, dw = B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none")
    assert torch.equal(B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none", (False, True))[1], dw)
    assert torch.equal(B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none", (True, False))[0], dh)
    B().operators_status()
    used, h, w, t, logits, lse64, _, off = definition(hidden, weight, targets)
    count, g = t.numel(), grad[used].double()[:, None]
    each = torch.arange(count, device="cuda")
    p = torch.exp(logits - lse64[:, None])
    G = g * p
    G[each, t] -= g[:, 0]
    # before the rounding: as in test_gpu_cross_entropy.py
    dG = g.abs() * p * (2 * off + SUM + 2 * U * lse64.abs() + 4 * U)[:, None] + 3 * U * G.abs()
    dG[each, t] += 2 * U * g[:, 0].abs()
    del logits, p
    # a common factor brings the largest near 1 (bf16) or 2^14 (fp16); a value that near a border may go to either side
    up = 2.0 ** ((14 if dtype == torch.float16 else 0) - math.floor(math.log2(g.abs().max().item())))

    def rounded(x):
        return (x * up).to(dtype).double() / up

    once, half = rounded(G), HALF[dtype]
    dG += torch.where(rounded(G - dG) == rounded(G + dG), 0.0, 2 * half * G.abs())
    dG[each, t] += half * half * G[each, t].abs()  # in two parts
    exact = once.clone()
    exact[each, t] = G[each, t]
    bound_h = dG @ w.abs() + ((v / 8 + 8) + 300) * 2.0 ** -23 * (G.abs() @ w.abs())
    bound_w = dG.t() @ h.abs() + (count / 8 + 8) * 2.0 ** -23 * (G.abs().t() @ h.abs())
    want_h, want_w = exact @ w, exact.t() @ h
    # the targets' entries rounded like the others  (fp32 sums over many classes may be as far off as fp16's half step)
    assert not inside((once.t() @ h).to(dtype), want_w, bound_w, dtype)
    if v / 8 * 2.0 ** -23 < half / 4:
        assert not inside((once @ w).to(dtype), want_h, bound_h, dtype)
    assert inside(dh[used], want_h, bound_h, dtype)
    assert inside(dw, want_w, bound_w, dtype)


@pytest.mark.parametrize("n,d,v,near", [(5000, 300, 9001, 700), (5000, 300, 9001, 1), (700, 72, 5003, 300), (9000, 24, 300000, 5000), (130, 600, 40000, 3),
                                          (200000, 16, 600, 600)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_targets_that_lie_together(n, d, v, near, dtype):
    """Many tokens for few tiles of classes, in any order, the last class among them."""
    hidden, weight, targets = inputs(n, d, v, dtype, 7, size=0.05)
    targets = v - 1 - targets % near
    grad = grads(n)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dh, dw = B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none")
    for _ in range(3):
        assert torch.equal(B().cross_entropy_backward(grad, hidden, weight, targets, lse, -100, "none")[1], dw)
    h, w = hidden.double(), weight.double()
    G = torch.softmax(h @ w.t(), 1)
    G[torch.arange(n), targets] -= 1
    G *= grad.double()[:, None]
    # the 2-norm of the errors: the results' own roundings, uniform within half a step (at most: over the square root of three), and
    # a tenth more for the roundings of the other entries of the logits' gradient
    for got, want in ((dh, G @ w), (dw, G.t() @ h)):
        assert (got.double() - want).norm() <= 1.1 * HALF[dtype] / 3 ** 0.5 * want.norm()
    B().operators_status()


# Roundings to nearest average out over many tokens, and their number grows with the depth of a sum only below its size; what is cut off
# adds up.  The mean loss is a few units off however many tokens there are: four of fp32, and sixteen for operands of 16 bits, whose
# own rounding is 2^12 to 2^15 units.
@pytest.mark.parametrize("n,d,v,dtype,most", [(1003, 509, 10007, torch.float32, 4 * U), (700, 2048, 5000, torch.float32, 4 * U),
                                              (2048, 1024, 20000, torch.bfloat16, 16 * U), (2048, 4096, 8000, torch.float16, 16 * U)])
def test_the_mean_loss_is_not_biased(n, d, v, dtype, most):
    hidden, weight, targets = inputs(n, d, v, dtype, 1)
    hidden = (hidden.float() + 1.5 * weight.float()[targets]).to(dtype)  # losses of about two
    want = definition(hidden, weight, targets)[6].mean()
    got = B().cross_entropy_forward(hidden, weight, targets)[0].double()
    assert abs(got - want) <= most * want


@pytest.mark.parametrize("n", [3000, 2 ** 17])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_sums_over_many_tokens_are_not_cut(n, dtype):
    """The layer's gradient from contributions of one sign, as many as there are tokens: on average over its entries it is a small part
    of the result's half step off, however many."""
    d, v = 96, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    hidden = ((torch.rand(n, d, device="cuda", generator=g) + 0.5) * torch.exp2(torch.rand(d, device="cuda", generator=g))).to(dtype)
    weight, targets = torch.zeros(v, d, device="cuda", dtype=dtype), torch.randint(0, v // 2, (n,), device="cuda", generator=g)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dw = B().cross_entropy_backward(torch.full((n,), 2.0 ** -10, device="cuda"), hidden, weight, targets, lse, -100, "none")[1]
    # all classes are as likely: 1 / 32, which is exact
    G = torch.full((n, v), 2.0 ** -15, dtype=torch.float64, device="cuda")
    G[torch.arange(n), targets] -= 2.0 ** -10
    want = G.t() @ hidden.double()
    off = (dw.double() - want) / want
    for rows in (off[:v // 2], off[v // 2:]):
        assert rows.mean().abs() <= HALF[dtype] / 4


@pytest.mark.parametrize("d", [64, 512, 4096])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_row_of_the_logits_gradient_adds_up_to_zero(d, dtype):
    """Logits of 30 from products of one sign.  A further column holds ones for the classes and zeros for the tokens: the gradient of
    the tokens' part of it is the sum of the logits' gradient over the classes."""
    n, v = 700, 300
    g = torch.Generator(device="cuda").manual_seed(4)
    hidden = torch.rand(n, d, device="cuda", generator=g) + 0.5
    weight = (torch.rand(v, d, device="cuda", generator=g) + 0.5) * (30 / d)
    hidden = torch.cat((hidden, torch.zeros(n, 1, device="cuda")), 1).to(dtype)
    weight = torch.cat((weight, torch.ones(v, 1, device="cuda")), 1).to(dtype)
    targets = torch.randint(0, v, (n,), device="cuda", generator=g)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    dh = B().cross_entropy_backward(torch.ones(n, device="cuda"), hidden, weight, targets, lse, -100, "none")[0]
    # on average: the roundings of a row's 300 entries, and of lse, which is 36: two units of it
    assert dh[:, -1].double().mean().abs() <= (HALF[dtype] / 16 if dtype != torch.float32 else 2 * 36 * U)


def sure(size, dtype, n=40, v=300, d=16):
    """Tokens that are as good as certain of their targets: logits of +size and -size, exactly."""
    g = torch.Generator(device="cuda").manual_seed(5)
    targets = torch.randint(0, d, (n,), device="cuda", generator=g)
    hidden, weight = torch.zeros(n, d, device="cuda"), torch.full((v, d), -1.0, device="cuda")
    hidden[torch.arange(n), targets] = size
    weight[:d] += 2 * torch.eye(d, device="cuda")
    return hidden.to(dtype), weight.to(dtype), targets


@pytest.mark.parametrize("size", [20.0, 92.0, 500.0, 6000.0])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_loss_of_a_sure_token(size, n, dtype):
    hidden, weight, targets = sure(size, dtype, n)
    size = hidden.amax().item()
    losses, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    assert (lse.double() - size).abs().max() <= 2 * U * size
    # the exponential of about 0 (2^-22) and the rounding of the sum: nothing that grows with the logits
    assert losses.abs().max() <= 2.0 ** -22 + 2 * U


@pytest.mark.parametrize("size", [20.0, 92.0, 500.0, 6000.0])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_gradient_of_a_sure_token(size, n, dtype):
    """lse is the target's logit, exactly: a probability of 1 and others of 0, so gradients of 0."""
    hidden, weight, targets = sure(size, dtype, n)
    lse = hidden.amax(1).float()
    dh, dw = B().cross_entropy_backward(torch.ones(n, device="cuda"), hidden, weight, targets, lse, -100, "none")
    # the exponential of 0 (2^-22), times a weight of 1; of `size` for the layer, n tokens of which may have one target
    assert dh.double().abs().max() <= 2.0 ** -22 + 2 * U
    assert dw.double().abs().max() <= (2.0 ** -22 + 2 * U) * n * hidden.amax().item()
