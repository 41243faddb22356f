"""Softmax cross entropy of a linear layer, both directions, against 64-bit formulas."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def B():
    from paper_2306_06098_b200 import binding
    return binding


def inputs(n, d, v, dtype, seed=0, labelled=1.0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    weight = torch.randn(v, d, device="cuda", generator=g) * (size * 2 / d ** 0.5)
    targets = torch.randint(0, v, (n,), device="cuda", generator=g)
    hidden = torch.randn(n, d, device="cuda", generator=g) + weight[targets]
    targets[torch.rand(n, device="cuda", generator=g) >= labelled] = -100
    return hidden.to(dtype), weight.to(dtype), targets


def definition(hidden, weight, targets, ignore=-100):
    """Rows that count, their logits, lse and losses in 64 bits, and how far fp32 sums of exact products may be off
    (one unit of 2^-23 of what has been added up, for each group of eight products; fp32 operands come in six
    products of parts and leave out less than 2^-22)."""
    used = targets != ignore
    h, w, t = hidden[used].double(), weight.double(), targets[used]
    logits = h @ w.t()
    size = h.abs() @ w.abs().t()
    groups = hidden.shape[-1] / 8 + 8
    off = ((6 * groups + 2 if hidden.dtype == torch.float32 else groups) * 2.0 ** -23 * size).amax(1)
    lse = torch.logsumexp(logits, 1)
    return used, h, w, t, logits, lse, lse - logits.gather(1, t[:, None])[:, 0], off


# the exponentials (2 units, and 3 units of an argument of up to 100), their sums: relative to the sum of exponentials
SUM = (4 + 3 * 100 + 50) * U


def check_forward(hidden, weight, targets, ignore=-100):
    used, _, _, _, _, lse64, loss64, off = definition(hidden, weight, targets, ignore)
    losses, lse = B().cross_entropy_forward(hidden, weight, targets, ignore, "none")
    assert losses.shape == lse.shape == targets.shape and losses.dtype == lse.dtype == torch.float32
    assert (losses[~used] == 0).all() and (lse[~used] == 0).all()
    assert ((lse[used].double() - lse64).abs() <= off + SUM + 2 * U * lse64.abs()).all()
    assert ((losses[used].double() - loss64).abs() <= 2 * off + SUM + 4 * U * (lse64.abs() + loss64.abs())).all()
    n = int(used.sum())
    for how in ("sum", "mean"):
        one, lse2 = B().cross_entropy_forward(hidden, weight, targets, ignore, how)
        assert torch.equal(lse2, lse) and one.shape == ()
        want = losses.double().sum() / (n if how == "mean" else 1)
        if n or how == "sum":
            assert abs(one.item() - want.item()) <= 2 * U * losses.double().abs().sum().item() / (n if how == "mean" else 1)
        else:
            assert one.isnan()
    again = B().cross_entropy_forward(hidden, weight, targets, ignore, "none")
    assert torch.equal(again[0], losses) and torch.equal(again[1], lse)
    B().operators_status()
    return losses, lse


def check_backward(hidden, weight, targets, grad, ignore=-100, reduction="none"):
    used, h, w, t, logits, lse64, _, off = definition(hidden, weight, targets, ignore)
    _, lse = B().cross_entropy_forward(hidden, weight, targets, ignore, reduction)
    dh, dw = B().cross_entropy_backward(grad, hidden, weight, targets, lse, ignore, reduction)
    assert dh.shape == hidden.shape and dw.shape == weight.shape and dh.dtype == dw.dtype == hidden.dtype
    n = int(used.sum())
    g = {"none": lambda: grad[used].double(), "sum": lambda: grad.double().expand(n),
         "mean": lambda: grad.double().expand(n) / max(1, n)}[reduction]()
    p = torch.exp(logits - lse64[:, None])
    del logits
    one = torch.zeros_like(p)
    one[torch.arange(n, device="cuda"), t] = 1
    G = g[:, None] * (p - one)
    half = {torch.float32: 2.0 ** -23, torch.bfloat16: HALF[torch.bfloat16], torch.float16: HALF[torch.float16]}[hidden.dtype]
    dG = g.abs()[:, None] * (p * (2 * off + SUM + 2 * U * lse64.abs() + 4 * U)[:, None] + 2 * U * one) + (half + 3 * U) * G.abs()
    if n:  # a probability below fp32's normal range, 2^-126, may be taken for 0 (exponentials are flushed there)
        dG = dG + g.abs()[:, None] * 2.0 ** -126
    if hidden.dtype == torch.float16 and n:  # what is left of values below fp16's range, next to the largest factor
        dG = dG + g.abs().max() * 2.0 ** -24 * 2.0 ** -13
    tiny = TINY[hidden.dtype]
    six = 6 if hidden.dtype == torch.float32 else 1

    def near(got, want, bound):
        assert ((got.double() - want).abs() <= bound + HALF[hidden.dtype] * (want.abs() + bound) + tiny).all()

    assert (dh[~used] == 0).all()
    near(dh[used], G @ w, dG @ w.abs() + (six * (w.shape[0] / 8 + 8) + 300) * 2.0 ** -23 * (G.abs() @ w.abs()))
    near(dw, G.t() @ h, dG.t() @ h.abs() + six * (n / 8 + 8) * 2.0 ** -23 * (G.abs().t() @ h.abs()))
    for want in ((True, False), (False, True)):
        part = B().cross_entropy_backward(grad, hidden, weight, targets, lse, ignore, reduction, want)
        assert (part[0] is not None, part[1] is not None) == want
        assert torch.equal(part[0], dh) if want[0] else torch.equal(part[1], dw)
    B().operators_status()
    return dh, dw


def grads(n, seed=9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, device="cuda", generator=g)


SIZES = [(1, 8, 64), (1, 1, 1), (2, 7, 2), (3, 64, 63), (127, 65, 256), (128, 100, 257), (129, 256, 1000),
         (5, 768, 30522), (300, 72, 513), (1000, 333, 777), (260, 520, 2050), (1, 2048, 130), (700, 16, 5)]


@pytest.mark.parametrize("n,d,v", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_sizes(n, d, v, dtype):
    check_forward(*inputs(n, d, v, dtype))


@pytest.mark.parametrize("n,d,v", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_sizes(n, d, v, dtype):
    hidden, weight, targets = inputs(n, d, v, dtype, labelled=0.8 if n > 3 else 1.0)
    check_backward(hidden, weight, targets, grads(n))
    check_backward(hidden, weight, targets, torch.tensor(0.7, device="cuda"), reduction="mean")
    check_backward(hidden, weight, targets, torch.tensor(-1e-3, device="cuda"), reduction="sum")


@pytest.mark.parametrize("labelled", [0.0, 0.01, 0.15, 0.5])
@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_without_a_target(labelled, dtype):
    hidden, weight, targets = inputs(515, 96, 1030, dtype, 3, labelled)
    losses, lse = check_forward(hidden, weight, targets)
    dh, dw = check_backward(hidden, weight, targets, grads(515))
    # whatever their hidden states hold
    bad = hidden.clone()
    bad[targets == -100] = float("nan")
    bad[targets == -100, 0] = float("inf")
    got = B().cross_entropy_forward(bad, weight, targets, -100, "none")
    assert torch.equal(got[0], losses) and torch.equal(got[1], lse)
    got = B().cross_entropy_backward(grads(515), bad, weight, targets, lse, -100, "none")
    assert torch.equal(got[0], dh) and torch.equal(got[1], dw)


def test_another_ignored_index():
    hidden, weight, targets = inputs(200, 64, 300, torch.bfloat16, 5)
    for ignore in (7, 299, -1, 2 ** 40):
        targets[::3] = ignore
        check_forward(hidden, weight, targets, ignore)
        check_backward(hidden, weight, targets, grads(200), ignore)


@pytest.mark.parametrize("dtype", TYPES)
def test_targets_out_of_range_are_told(dtype):
    hidden, weight, targets = inputs(40, 32, 100, dtype, 6)
    for bad in (100, -1, 2 ** 40, -2 ** 62):
        t = targets.clone()
        t[11] = bad
        losses, lse = B().cross_entropy_forward(hidden, weight, t, -100, "none")
        assert losses[11].isnan() and losses.isnan().sum() == 1 and not lse.isnan().any()
        assert B().cross_entropy_forward(hidden, weight, t)[0].isnan()
        dh, dw = B().cross_entropy_backward(grads(40), hidden, weight, t, lse, -100, "none")
        assert dh[11].isnan().all() and dh.isnan().any(1).sum() == 1 and dw.isnan().all()


def test_values_that_are_not_finite():
    hidden, weight, targets = inputs(40, 32, 100, torch.float32, 6)
    hidden[3, 2] = float("nan")
    losses, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    assert losses[3].isnan() and lse[3].isnan() and losses.isnan().sum() == 1
    weight[7] = float("nan")
    assert B().cross_entropy_forward(hidden, weight, targets, -100, "none")[0].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_large_logits(dtype):
    """Probabilities of 0 and 1: the largest logits reach 100, where a row's exponentials span fp32's range."""
    hidden, weight, targets = inputs(150, 64, 400, dtype, 8, size=8.0)
    check_forward(hidden, weight, targets)
    check_backward(hidden, weight, targets, grads(150))


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    hidden, weight, targets = inputs(6 * 35, 96, 200, dtype, 4)
    want = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    h3, t3 = hidden.view(6, 35, 96), targets.view(6, 35)
    wide = torch.empty(6, 35, 101, dtype=dtype, device="cuda")
    odd = torch.empty(200 * 96 + 1, dtype=dtype, device="cuda")[1:].view(200, 96)
    odd.copy_(weight)
    padded = torch.empty(200, 97, dtype=dtype, device="cuda")[:, 1:]
    padded.copy_(weight)
    eight = torch.empty(200, 104, dtype=dtype, device="cuda")[:, :96]
    eight.copy_(weight)
    wide[..., 3:99] = h3
    grad = grads(6 * 35).view(6, 35)
    back = B().cross_entropy_backward(grad, h3, weight, t3, want[1].view(6, 35), -100, "none")
    for h in (h3, wide[..., 3:99], h3.transpose(0, 1).contiguous().transpose(0, 1)):
        for w in (weight, odd, padded, eight, weight.t().contiguous().t()):
            for t in (t3, t3.t().contiguous().t()):
                losses, lse = B().cross_entropy_forward(h, w, t, -100, "none")
                assert torch.equal(losses.view(-1), want[0]) and torch.equal(lse.view(-1), want[1])
            for g in (grad, grad.t().contiguous().t()):
                got = B().cross_entropy_backward(g, h, w, t3, lse, -100, "none")
                assert torch.equal(got[0], back[0]) and torch.equal(got[1], back[1])
    one = torch.tensor(2.0, device="cuda").expand(6, 35)
    a = B().cross_entropy_backward(one, h3, weight, t3, lse, -100, "none")
    b = B().cross_entropy_backward(one.contiguous(), h3, weight, t3, lse, -100, "none")
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_one_token_without_other_dimensions_and_no_tokens():
    hidden, weight, targets = inputs(1, 40, 90, torch.bfloat16, 2)
    a = B().cross_entropy_forward(hidden[0], weight, targets[0], -100, "none")
    assert a[0].shape == () and torch.equal(a[0], B().cross_entropy_forward(hidden, weight, targets, -100, "none")[0][0])
    h, t = torch.empty(0, 40, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    w = weight.float()
    losses, lse = B().cross_entropy_forward(h, w, t, -100, "none")
    assert losses.shape == lse.shape == (0,)
    assert B().cross_entropy_forward(h, w, t, -100, "sum")[0] == 0 and B().cross_entropy_forward(h, w, t)[0].isnan()
    dh, dw = B().cross_entropy_backward(torch.ones((), device="cuda"), h, w, t, lse)
    assert dh.shape == (0, 40) and (dw == 0).all()


@pytest.mark.parametrize("dtype,n,v", [(torch.bfloat16, 16500, 20100), (torch.float16, 40000, 5000), (torch.float32, 9000, 12000)])
def test_several_pieces_of_the_vocabulary(dtype, n, v):
    hidden, weight, targets = inputs(n, 72, v, dtype, 3, 0.5)
    check_backward(hidden, weight, targets, torch.tensor(1.0, device="cuda"), reduction="mean")


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e6])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_of_any_size(dtype, scale):
    hidden, weight, targets = inputs(140, 64, 300, dtype, 3)
    check_backward(hidden, weight, targets, grads(140) * scale)
    dh, dw = check_backward(hidden, weight, targets, torch.zeros(140, device="cuda"))
    assert (dh == 0).all() and (dw == 0).all()


def test_factors_of_fp16_that_differ():
    hidden, weight, targets = inputs(140, 64, 300, torch.float16, 3)
    check_backward(hidden, weight, targets, grads(140) * torch.logspace(-3, 3, 140, device="cuda"))


# ------------------------------------------------------------------ autograd, streams, graphs
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd(reduction):
    from paper_2306_06098_b200.loss import LinearCrossEntropy, linear_cross_entropy
    hidden, weight, targets = inputs(5 * 33, 48, 350, torch.float32, 4, 0.8)
    hidden, targets = hidden.view(5, 33, 48).requires_grad_(True), targets.view(5, 33)
    layer = LinearCrossEntropy(48, 350, torch.nn.Parameter(weight), reduction=reduction)
    value = layer(hidden, targets)
    factor = torch.randn(value.shape, device="cuda")
    (value * factor).sum().backward()
    h64, w64 = hidden.detach().double().requires_grad_(True), weight.double().requires_grad_(True)
    want = torch.nn.functional.cross_entropy((h64 @ w64.t()).transpose(1, 2), targets, reduction=reduction)
    (want * factor).sum().backward()
    assert (value - want).abs().max() <= 1e-5 * want.abs().max()
    for a, b in ((hidden.grad, h64.grad), (layer.weight.grad, w64.grad)):
        assert (a - b).norm() <= 2e-5 * b.norm()
    with torch.no_grad():
        assert torch.equal(linear_cross_entropy(hidden, weight, targets, -100, reduction), value)
    frozen = linear_cross_entropy(hidden, weight, targets, -100, reduction)
    (frozen * factor).sum().backward()
    with pytest.raises(ValueError):
        LinearCrossEntropy(48, 350, reduction="median")
    with pytest.raises(ValueError):
        LinearCrossEntropy(47, 350, layer.weight)


def test_gradient_against_differences():
    from paper_2306_06098_b200.loss import linear_cross_entropy
    hidden, weight, targets = inputs(6, 10, 20, torch.float32, 4)
    hidden.requires_grad_(True)
    weight.requires_grad_(True)
    gh, gw = torch.autograd.grad(linear_cross_entropy(hidden, weight, targets, reduction="sum"), (hidden, weight))
    step = 2.0 ** -6
    with torch.no_grad():
        for leaf, grad, places in ((hidden, gh, range(0, 60, 7)), (weight, gw, range(0, 200, 23))):
            for i in places:
                e = torch.zeros(leaf.numel(), device="cuda")
                e[i] = step
                e = e.view(leaf.shape)
                up = linear_cross_entropy(hidden + e if leaf is hidden else hidden, weight + e if leaf is weight else weight,
                                          targets, reduction="none").double().sum().item()
                down = linear_cross_entropy(hidden - e if leaf is hidden else hidden, weight - e if leaf is weight else weight,
                                            targets, reduction="none").double().sum().item()
                # third derivatives: a logit moves by e times a value of up to 6, a cumulant of it is below 6^3 a
                # token; rounding: six losses of up to 30 with 20 units each
                assert abs((up - down) / (2 * step) - grad.view(-1)[i].item()) < 6 * 6 ** 3 * step ** 2 / 6 + 6 * 30 * 20 * U / step


def test_captured_and_on_other_streams():
    hidden, weight, targets = inputs(300, 128, 1000, torch.bfloat16, 4, 0.7)
    other = inputs(300, 128, 1000, torch.bfloat16, 5, 0.3)
    one = torch.ones((), device="cuda")

    def both(h, w, t):
        value, lse = B().cross_entropy_forward(h, w, t)
        return (value, *B().cross_entropy_backward(one, h, w, t, lse))

    want, want2 = both(hidden, weight, targets), both(*other)
    h, w, t = hidden.clone(), weight.clone(), targets.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = both(h, w, t)
    for _ in range(2):
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for a, b in zip((h, w, t), other):
            a.copy_(b)
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want2))
        for a, b in zip((h, w, t), (hidden, weight, targets)):
            a.copy_(b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = []
    for _ in range(4):
        for s, data in zip(streams, ((hidden, weight, targets), other)):
            with torch.cuda.stream(s):
                results.append(both(*data))
    torch.cuda.synchronize()
    for k, r in enumerate(results):
        assert all(torch.equal(a, b) for a, b in zip(r, want2 if k % 2 else want))
    lone = B().cross_entropy_forward(hidden, weight, targets, stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(lone[0], want[0])
    B().operators_status()


# ------------------------------------------------------------------ a few tokens
@pytest.mark.parametrize("n", [1, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("d,v", [(24, 1), (100, 31), (129, 33), (768, 2000), (1300, 513), (2048, 700), (2056, 100), (4096, 300),
                                 (4100, 65), (8000, 40)])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_tokens(n, d, v, dtype):
    hidden, weight, targets = inputs(n, d, v, dtype, 4)
    check_forward(hidden, weight, targets)
    check_backward(hidden, weight, targets, grads(n))
    if n > 1:  # rows of wider tensors, and a token that does not count, whatever it holds
        targets[1] = -100
        hidden, weight = (torch.nn.functional.pad(x, (1, 2))[:, 1:-2] for x in (hidden, weight))
        hidden[1] = float("nan")
        losses, _ = check_forward(hidden, weight, targets)
        assert not losses.isnan().any()
        dh, dw = B().cross_entropy_backward(torch.tensor(2.0, device="cuda"), hidden, weight, targets,
                                            B().cross_entropy_forward(hidden, weight, targets)[1])
        assert not dh.isnan().any() and not dw.isnan().any() and (dh[1] == 0).all()


@pytest.mark.parametrize("n", [2, 7])
def test_few_tokens_that_have_no_target_or_a_wrong_one(n):
    hidden, weight, targets = inputs(n, 72, 300, torch.bfloat16, 5)
    one = torch.ones((), device="cuda")
    targets[0] = 300
    losses, lse = B().cross_entropy_forward(hidden, weight, targets, -100, "none")
    assert losses[0].isnan() and not losses[1:].isnan().any() and not lse.isnan().any()
    dh, dw = B().cross_entropy_backward(one, hidden, weight, targets, lse, -100, "sum")
    assert dh[0].isnan().all() and dw.isnan().all() and not dh[1:].isnan().any()
    targets[:] = 0  # a class that does not count
    for how in ("none", "sum", "mean"):
        got, lse = B().cross_entropy_forward(hidden, weight, targets, 0, how)
        assert got.isnan() if how == "mean" else (got == 0).all()
        dh, dw = B().cross_entropy_backward(torch.ones_like(got), hidden, weight, targets, lse, 0, how)
        assert (dh == 0).all() and (lse == 0).all() and (dw == 0).all()


# ------------------------------------------------------------------ wider pieces where few tokens count
@pytest.mark.parametrize("labelled", [0.0, 0.0001, 0.1, 0.2, 0.45, 0.9])
@pytest.mark.parametrize("dtype,v", [(torch.float32, 5003), (torch.bfloat16, 9001), (torch.float16, 8192)])
def test_pieces_of_every_width(labelled, dtype, v):
    n, d = 16300, 40  # pieces of 1280 columns for fp32, 4096 for 16 bits, when all tokens count
    hidden, weight, targets = inputs(n, d, v, dtype, 6, labelled)
    check_backward(hidden, weight, targets, grads(n))
    check_backward(hidden, weight, targets, torch.tensor(0.5, device="cuda"), reduction="sum")
