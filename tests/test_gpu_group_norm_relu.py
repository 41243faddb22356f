"""Group norm's backward pass through relu, in every type and access width, on chip and streamed, and
gradients that are not finite at positions whose relu is off."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)
HALF_ULP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}
EPS = 1e-5

# 16-, 4- and 2-byte accesses of the half types, 16 and 4 of fp32; on chip in one block and in
# clusters, streamed
SIZES = [(2, 16, 4, (8, 8)), (1, 30, 6, (7, 5)), (3, 33, 11, (9, 9)), (2, 64, 32, (56, 56)), (4, 130, 26, (20, 20)),
         (1, 128, 32, (130, 130)), (2, 130, 26, (128, 128)), (1, 65, 13, (200, 160))]


def rand(shape, seed, dtype=torch.float32, mean=0.0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (mean + size * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def inputs(n, c, pos, dtype, seed):
    return rand((n, *pos, c), seed, dtype).permute(0, len(pos) + 1, *range(1, len(pos) + 1))


def problem(size, dtype):
    n, c, groups, pos = size
    x, dy = inputs(n, c, pos, dtype, 3), inputs(n, c, pos, dtype, 4)
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    v = x.double().reshape(n, groups, -1)
    m = v.mean(2, keepdim=True)
    r = 1.0 / ((v - m).square().mean(2, keepdim=True) + EPS).sqrt()
    h = ((v - m) * r).reshape(x.shape)
    shape = (1, c) + (1,) * len(pos)
    z = h * w.double().reshape(shape) + b.double().reshape(shape)
    return x, dy, w, b, h, z, r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_backward_of_relu(size, dtype):
    from paper_2306_06098_b200 import binding as B
    n, c, groups, pos = size
    x, dy, w, b, h, z, r = problem(size, dtype)
    # relu's derivative jumps at 0: no gradient where fp32 cannot tell the side of z
    dy = torch.where(z.abs() < 1e-3, torch.zeros_like(dy), dy)
    _, mean, rstd = B.group_norm_forward(x, groups, w, b, EPS, "relu")
    dx, dw, db = B.group_norm_backward(dy, x, mean, rstd, groups, w, b, "relu")
    e = torch.where(z > 0, dy.double(), torch.zeros_like(z))
    ew = e * w.double().reshape((1, c) + (1,) * len(pos))
    size_of = math.prod(x.shape[1:]) // groups

    def joint(t):
        return t.reshape(n, groups, -1).mean(2, keepdim=True).expand(n, groups, size_of).reshape(x.shape)

    rr = r.expand(n, groups, size_of).reshape(x.shape)
    want = rr * (ew - joint(ew) - h * joint(ew * h))
    mag = rr * (ew.abs() + joint(ew.abs()) + h.abs() * joint((ew * h).abs()))
    # as for the other activations: h is off by 160 U of the largest |x| rstd of its group and 110 U
    # of itself, every term carries that once or twice
    tol = (400 + 400 * (x.double().abs().amax() * rstd.double().max()).item()) * U
    assert ((dx.double() - want).abs() <= tol * (mag + mag.mean()) + HALF_ULP[dtype] * want.abs() + TINY[dtype]).all()
    rest = (0,) + tuple(range(2, x.dim()))
    for got, ref, m in ((dw, (e * h).sum(rest), (e * h).abs().sum(rest)), (db, e.sum(rest), e.abs().sum(rest))):
        assert ((got.double() - ref).abs() <= tol * (m + m.mean())).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_what_a_dead_relu_receives_does_not_matter(size, dtype, bad):
    """The derivative there selects 0, whatever comes in: an overflowed gradient too."""
    from paper_2306_06098_b200 import binding as B
    n, c, groups, pos = size
    x, dy, w, b, _, z, _ = problem(size, dtype)
    off = z < -0.5
    assert off.any()
    _, mean, rstd = B.group_norm_forward(x, groups, w, b, EPS, "relu")
    want = B.group_norm_backward(torch.where(off, torch.zeros_like(dy), dy), x, mean, rstd, groups, w, b, "relu")
    got = B.group_norm_backward(torch.where(off, torch.full_like(dy, bad), dy), x, mean, rstd, groups, w, b, "relu")
    for p, q in zip(got, want):
        assert torch.equal(p, q) and p.isfinite().all()
