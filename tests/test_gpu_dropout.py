"""Dropout whose mask is computed from a counter: every element against the generator restated in numpy."""
import pytest
import torch

from philox import kept, threshold

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def B():
    from paper_2306_06098_b200 import binding
    return binding


def rand(shape, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", generator=g).to(dtype)


def check(x, p, rng=(3, 4), residual=None, state=None):
    y = B().dropout(x, p, rng if state is None else state, residual)
    assert y.shape == x.shape and y.dtype == x.dtype and y.is_contiguous()
    t = threshold(p)
    keep = kept(tuple(x.shape), p, *rng).cuda()
    s = x.double() * (65536 / (65536 - t) if t < 65536 else 0.0)
    want = torch.where(keep, s, 0.0)
    off = 2 * U * want.abs()  # the scale and the product
    if residual is not None:
        want = want + residual.double()
        off = off + U * want.abs()
    else:
        assert (y[~keep] == 0).all()
    assert ((y.double() - want).abs() <= off + HALF[x.dtype] * (want.abs() + off) + TINY[x.dtype]).all()
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (255,), (256,), (1000, 1), (3, 257), (517, 1001), (64, 768),
                                   (2, 3, 5, 7), (4096, 40)])
def test_every_element(shape, dtype):
    x = rand(shape, 1, dtype)
    check(x, 0.25)
    check(x, 0.1, (2 ** 64 - 1, 2 ** 63), rand(shape, 2, dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_the_mask_goes_by_the_logical_order(dtype):
    x = rand((24, 40, 56), 3, dtype)
    a = B().dropout(x, 0.5, (1, 2))
    for other in (x.permute(2, 0, 1).contiguous().permute(1, 2, 0),             # copied first
                  torch.cat((x, x), 2)[..., :56], torch.cat((x[..., :3], x), 2)[..., 3:],
                  torch.cat((x[:1], x))[1:], x.contiguous().view(-1)[0:].view(x.shape)):
        assert torch.equal(other, x)
        assert torch.equal(B().dropout(other, 0.5, (1, 2)), a)
    flat = torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:]  # not on 16 bytes
    flat.copy_(x.view(-1))
    assert torch.equal(B().dropout(flat, 0.5, (1, 2)), a.view(-1))
    assert torch.equal(B().dropout(x, 0.5, (1, 2), torch.zeros_like(x)[..., :1].expand_as(x)), a)


def test_shares_from_none_to_all():
    x = rand((777,), 1)
    assert torch.equal(B().dropout(x, 0.0, None), x)
    assert (B().dropout(x, 1.0, (1, 1)) == 0).all()
    assert torch.equal(B().dropout(x, 1.0, (1, 1), x), x)
    assert torch.equal(B().dropout(x, 2.0 ** -18, (1, 1)), x)  # rounds to none
    check(x, 1 - 2.0 ** -16)
    for shape in ((0,), (3, 0), (0, 5)):
        assert B().dropout(torch.empty(shape, device="cuda"), 0.5, (1, 1)).shape == shape


def test_bad_values_that_are_dropped_are_gone():
    x = rand((1000,), 1)
    keep = kept((1000,), 0.5, 3, 4).cuda()
    for bad in (float("nan"), float("inf")):
        y = B().dropout(torch.where(keep, x, torch.full_like(x, bad)), 0.5, (3, 4))
        assert torch.equal(y, B().dropout(x, 0.5, (3, 4)))


def test_the_state_on_the_device():
    x = rand((300, 96), 1, torch.bfloat16)
    state = torch.tensor([-5, 2 ** 40 + 9], device="cuda")
    check(x, 0.3, (-5, 2 ** 40 + 9), None, state)
    g = torch.cuda.CUDAGraph()
    B().dropout(x, 0.3, state)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        y = B().dropout(x, 0.3, state)
    for s in ((1, 2), (3, 2 ** 62)):
        state.copy_(torch.tensor(s))
        g.replay()
        assert torch.equal(y, B().dropout(x, 0.3, s))


def test_offsets_beyond_32_bits():
    """Rows of a broadcast row, checked at the ends."""
    n, d = 2 ** 20 + 1, 2 ** 12
    x = torch.ones(1, d, dtype=torch.bfloat16, device="cuda").expand(n, d)
    y = B().dropout(x, 0.5, (7, 8))
    for row in (0, 2 ** 19 - 1, 2 ** 19, 2 ** 20):
        assert torch.equal(y[row] != 0, kept((d,), 0.5, 7, 8, row * d).cuda())


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients(dtype):
    from paper_2306_06098_b200.dropout import dropout
    x, r, c = rand((33, 100), 1, dtype).requires_grad_(True), rand((33, 100), 2, dtype).requires_grad_(True), rand((33, 100), 3, dtype)
    state = torch.tensor([11, 12], device="cuda")
    y = dropout(x, 0.4, state, r)
    dx, dr = torch.autograd.grad(y, (x, r), c)
    assert torch.equal(dr, c) and torch.equal(dx, B().dropout(c, 0.4, (11, 12)))
    y = dropout(x, 0.4, state)
    state.add_(1)  # the mask of the other direction would be another one
    with pytest.raises(RuntimeError, match="modified"):
        torch.autograd.grad(y, x, c)
    y = dropout(x, 0.0, None, r)
    assert torch.equal(torch.autograd.grad(y, x, c)[0], c)


def test_module():
    from paper_2306_06098_b200.dropout import Dropout, new_rng, take
    torch.manual_seed(3)
    a, b = Dropout(0.5, device="cuda"), Dropout(0.5, device="cuda")
    assert a.rng[0] != b.rng[0]
    x = torch.ones(40, 50, device="cuda", requires_grad=True)
    y1, y2 = a(x), a(x)
    assert not torch.equal(y1, y2) and not torch.equal(y1, b(x))
    y1.sum().backward()
    assert torch.equal(x.grad, y1)
    c = Dropout(0.5, seed=0, device="cuda")
    c.load_state_dict(a.state_dict())
    assert torch.equal(c(x), a(x))
    a.eval()
    assert a(x) is x and torch.equal(a(x, x), 2 * x)
    with pytest.raises(ValueError):
        Dropout(1.5)
    s = new_rng(2 ** 64 - 1, "cuda")
    assert s.tolist() == [-1, 0] and take(s).tolist() == [-1, 0] and s.tolist() == [-1, 1]


@pytest.mark.parametrize("rows,d", [(1, 1), (3, 5), (1, 8), (7, 31), (513, 1001), (9001, 301), (3, 100003)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_one_behind_the_other(rows, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(rows, d, device="cuda", generator=g).to(dtype) for _ in range(2))
    for p in (0.0, 0.25, 1.0):
        for residual in (None, r):
            got = B().dropout(x, p, (9, 10), residual)
            # the same rows, further apart
            wide = [t if t is None else torch.nn.functional.pad(t, (0, 3))[:, :d] for t in (x, residual)]
            assert torch.equal(got, B().dropout(wide[0], p, (9, 10), wide[1]))
            keep = kept((rows, d), p, 9, 10).cuda() if p else torch.ones_like(x, dtype=torch.bool)
            want = torch.where(keep, x.float() * (65536 / (65536 - threshold(p)) if p < 1 else 0.0), 0.0)
            assert torch.equal(got, (want if residual is None else want + r.float()).to(dtype))
