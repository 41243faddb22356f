"""Group norm with an activation, channels last, both directions, against 64-bit formulas."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# rounding to a type, where that is coarser than the fp32 arithmetic: half its spacing above 1
HALF_ULP = {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2,
            torch.float16: torch.finfo(torch.float16).eps / 2}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}
ACTS = ("none", "relu", "silu")


def _binding():
    from paper_2306_06098_b200 import binding
    return binding


def rand(shape, seed, dtype=torch.float32, mean=0.0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (mean + size * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def inputs(n, c, pos, dtype, seed=0, mean=0.0, size=1.0, pad=0, front=0):
    """Channels last; pad / front: a channel slice of a wider tensor."""
    x = rand((n, *pos, c + pad + front), seed, dtype, mean, size)[..., front:front + c]
    return x.permute(0, len(pos) + 1, *range(1, len(pos) + 1))


def definition(x, groups, w, b, eps, act):
    """y, mean, rstd, z and h in 64 bits."""
    n, c = x.shape[:2]
    v = x.double().reshape(n, groups, -1)
    mean = v.mean(2, keepdim=True)
    rstd = 1.0 / ((v - mean).square().mean(2, keepdim=True) + eps).sqrt()
    h = ((v - mean) * rstd).reshape(x.shape)
    shape = (1, c) + (1,) * (x.dim() - 2)
    z = h
    if w is not None:
        z = z * w.double().reshape(shape)
    if b is not None:
        z = z + b.double().reshape(shape)
    y = {"none": z, "relu": z.clamp(min=0), "silu": z / (1 + torch.exp(-z))}[act]
    return y, mean[..., 0], rstd[..., 0], z, h


def check_forward(x, groups, w=None, b=None, eps=1e-5, act="none"):
    B = _binding()
    y, mean, rstd = B.group_norm_forward(x, groups, w, b, eps, act)
    assert y.shape == x.shape and y.dtype == x.dtype and mean.shape == rstd.shape == (x.shape[0], groups)
    want, m64, r64, z, h = definition(x, groups, w, b, eps, act)
    n, c = x.shape[:2]
    big = x.double().abs().reshape(n, groups, -1).amax(2)  # largest value of a group
    # a thread adds at most 64 differences, a few joins follow: mean within 160 U of the largest
    # value; M2 within 200 U of itself (and of what the mean's error adds)
    assert ((mean - m64).abs() <= 160 * U * big).all()
    assert ((rstd - r64).abs() <= r64 * 110 * U).all()
    group = (n, groups, 1)
    slack = (160 * U * big * r64).reshape(group)  # error of h from the mean's
    wa = torch.ones(c, dtype=torch.float64, device="cuda") if w is None else w.double().abs()
    ba = torch.zeros(c, dtype=torch.float64, device="cuda") if b is None else b.double().abs()
    shape = (1, c) + (1,) * (x.dim() - 2)
    wa, ba = wa.reshape(shape), ba.reshape(shape)
    err_h = slack.expand(n, groups, math.prod(x.shape[1:]) // groups).reshape(x.shape) + 128 * U * h.abs()
    bound = 1.1 * (wa * err_h + 16 * U * (z.abs() + ba)) + 8 * U * want.abs()
    bound = bound + HALF_ULP[x.dtype] * (want.abs() + bound) + TINY[x.dtype]
    assert ((y.double() - want).abs() <= bound + 1e-45).all()
    again = B.group_norm_forward(x, groups, w, b, eps, act)
    for p, q in zip((y, mean, rstd), again):  # repeats bit for bit
        assert torch.equal(p, q)
    return y, mean, rstd


def backward64(dy, x, groups, w, b, eps, act):
    """dx, dw, db by the formula in 64 bits, and the sums of absolute terms."""
    n, c = x.shape[:2]
    _, _, r, z, h = definition(x, groups, w, b, eps, act)
    d = {"none": torch.ones_like(z), "relu": (z > 0).double(),
         "silu": torch.sigmoid(z) * (1 + z * (1 - torch.sigmoid(z)))}[act]
    e = dy.double() * d
    shape = (1, c) + (1,) * (x.dim() - 2)
    ew = e if w is None else e * w.double().reshape(shape)
    rest = (0,) + tuple(range(2, x.dim()))

    def mean(t):
        return t.reshape(n, groups, -1).mean(2, keepdim=True).expand(
            n, groups, math.prod(x.shape[1:]) // groups).reshape(x.shape)

    rr = r.unsqueeze(2).expand(n, groups, math.prod(x.shape[1:]) // groups).reshape(x.shape)
    dx = rr * (ew - mean(ew) - h * mean(ew * h))
    size = rr * (ew.abs() + mean(ew.abs()) + h.abs() * mean((ew * h).abs()))
    return (dx, (e * h).sum(rest), e.sum(rest), size, (e * h).abs().sum(rest), e.abs().sum(rest))


def check_backward(dy, x, groups, w, b, eps, act):
    B = _binding()
    _, mean, rstd = B.group_norm_forward(x, groups, w, b, eps, act)
    dx, dw, db = B.group_norm_backward(dy, x, mean, rstd, groups, w, b, act)
    assert dx.shape == x.shape and dx.dtype == x.dtype
    want, w64, b64, size, wsize, bsize = backward64(dy, x, groups, w, b, eps, act)
    # h is off by 160 U of the largest |x| rstd of its group (mean) and 110 U of itself (rstd);
    # every term of dx and of the sums carries that once or twice, silu's derivative too
    n = x.shape[0]
    big = (x.double().abs().reshape(n, groups, -1).amax(2) * rstd.double()).max().item()
    tol = (400 + 400 * big) * U
    bound = tol * (size + size.mean()) + HALF_ULP[x.dtype] * want.abs() + TINY[x.dtype]
    assert ((dx.double() - want).abs() <= bound + 1e-45).all()
    for got, ref, mag, p in ((dw, w64, wsize, w), (db, b64, bsize, b)):
        if p is None:
            assert got is None
            continue
        assert got.dtype == p.dtype and got.shape == p.shape
        lim = tol * (mag + mag.mean()) + HALF_ULP[p.dtype] * ref.abs() + TINY[p.dtype]
        assert ((got.double() - ref).abs() <= lim + 1e-45).all()
    again = B.group_norm_backward(dy, x, mean, rstd, groups, w, b, act)
    for p, q in zip((dx, dw, db), again):
        assert p is q or torch.equal(p, q)
    return dx, dw, db


# (n, channels, groups, positions): one value, one row, odd sizes, groups of 1 to thousands of channels,
# rows from one to many, samples from one to many, sizes around the blocks' limits
SIZES = [
    (1, 1, 1, (1,)), (1, 8, 8, (1,)), (3, 7, 7, (5,)), (2, 6, 3, (1, 1)), (5, 16, 8, (8, 8)),
    (4, 16, 4, (32, 32)), (2, 64, 32, (56, 56)), (1, 512, 32, (7, 7)), (3, 120, 24, (37, 53)),
    (2, 185, 37, (9, 4)), (1, 1030, 1, (3, 5)), (2, 4100, 2, (2, 3)), (1, 2050, 2050, (4,)),
    (1, 8200, 1, (3,)), (1, 24, 3, (129, 127)), (300, 32, 2, (2, 2)), (1, 2, 1, (100_003,)),
    (1, 4104, 513, (2, 2)), (2, 36, 18, (3, 3, 3)), (1, 40, 5, (70_001,)), (1000, 48, 12, (1,)),
    (1, 264, 1, (300,)), (7, 320, 32, (16, 16)), (2, 1, 1, (4097,)), (16, 64, 8, (64, 64)),
    (1, 128, 32, (130, 130)), (3, 72, 9, (33, 31)),
]


@pytest.mark.parametrize("dtype", list(HALF_ULP))
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype):
    n, c, groups, pos = size
    act = ACTS[(c + n) % 3]
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    check_forward(inputs(n, c, pos, dtype, 3, mean=0.5), groups, w, b, act=act)


# where the cut into tiles and blocks changes: many samples of few rows (wide tiles), few samples
# (narrow ones), odd channel counts whose columns do not fill the threads, samples too large to stay on chip
CUTS = [
    (600, 96, 12, (1,)), (500, 200, 8, (2, 3)), (450, 130, 26, (3, 3)), (460, 185, 37, (4,)),
    (445, 64, 8, (8, 8)), (1, 35, 7, (40, 53)), (2, 33, 11, (100, 30)), (1, 256, 32, (14, 14)),
    (4, 185, 37, (50, 50)), (2, 130, 26, (128, 128)), (1, 1260, 42, (60, 60)),
    (2, 320, 32, (160, 160)), (3, 65, 13, (200, 160)),
]


@pytest.mark.parametrize("dtype", list(HALF_ULP))
@pytest.mark.parametrize("size", CUTS)
def test_where_the_work_is_cut_differently(size, dtype):
    n, c, groups, pos = size
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    x = inputs(n, c, pos, dtype, 3, mean=0.5)
    check_forward(x, groups, w, b, act="silu")
    check_backward(inputs(n, c, pos, dtype, 4), x, groups, w, b, 1e-3, "silu")


def away_from_the_jump(x, groups, w, b, eps):
    """relu's derivative jumps at z = 0: values of x whose z is too near for fp32 to tell the side
    are moved until there are none."""
    for _ in range(20):
        z = definition(x, groups, w, b, eps, "relu")[3]
        near = z.abs() < 2e-3
        if not near.any():
            return x
        x = torch.where(near, (x.double() + 0.05 * (1 + x.double().abs())).to(x.dtype), x)
    return x


@pytest.mark.parametrize("dtype", list(HALF_ULP))
@pytest.mark.parametrize("size", SIZES)
def test_backward(size, dtype):
    n, c, groups, pos = size
    act = ("none", "silu")[(c + n) % 2]
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    x = inputs(n, c, pos, dtype, 3, mean=0.5)
    check_backward(inputs(n, c, pos, dtype, 4), x, groups, w, b, 1e-3, act)


@pytest.mark.parametrize("size", [(2, 16, 4, (8, 8)), (1, 30, 6, (7, 5)), (2, 32, 32, (20, 20))])
def test_backward_of_relu(size):
    n, c, groups, pos = size
    w, b = rand((c,), 1, mean=1.0, size=0.1), rand((c,), 2, size=0.3)
    x = away_from_the_jump(inputs(n, c, pos, torch.float32, 3), groups, w, b, 1e-5)
    assert (definition(x, groups, w, b, 1e-5, "relu")[3].abs() >= 1e-4).all()
    check_backward(inputs(n, c, pos, torch.float32, 4), x, groups, w, b, 1e-5, "relu")


@pytest.mark.parametrize("dtype", list(HALF_ULP))
@pytest.mark.parametrize("pad,front", [(1, 0), (8, 8), (0, 3), (2, 2), (24, 4)])
def test_channel_slices(dtype, pad, front):
    n, c, groups, pos = 3, 40, 8, (11, 13)
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    x = inputs(n, c, pos, dtype, 3, pad=pad, front=front)
    dy = inputs(n, c, pos, dtype, 4, pad=front, front=pad)
    check_forward(x, groups, w, b, act="silu")
    check_backward(dy, x, groups, w, b, 1e-5, "silu")


def test_other_layouts():
    n, c, groups = 2, 12, 4
    w, b = rand((c,), 1, mean=1.0, size=0.3), rand((c,), 2, size=0.3)
    wide = rand((n, c, 10, 9), 3)
    for x in (wide, wide.transpose(2, 3), wide[:, :, 1:8:2, 2:7], wide[:1].expand(3, c, 10, 9),
              wide.contiguous(memory_format=torch.channels_last)[:, :, 2:9, 1:8],
              inputs(n, c, (6,), torch.float32, 5)[::2], wide[:, :, :1, :1], wide[:, :, 0, 0]):
        check_forward(x, groups, w, b)
        check_backward(rand((), 6).expand(x.shape), x, groups, w, b, 1e-5, "silu")


@pytest.mark.parametrize("pdtype", list(HALF_ULP))
@pytest.mark.parametrize("dtype", list(HALF_ULP))
def test_parameter_types_and_absence(pdtype, dtype):
    n, c, groups, pos = 2, 32, 8, (9, 9)
    w, b = rand((c,), 1, pdtype, 1.0, 0.3), rand((c,), 2, pdtype, 0.0, 0.3)
    x, dy = inputs(n, c, pos, dtype, 3), inputs(n, c, pos, dtype, 4)
    for ww, bb in ((w, b), (w, None), (None, b), (None, None)):
        check_forward(x, groups, ww, bb, act="silu")
        check_backward(dy, x, groups, ww, bb, 1e-5, "silu")


@pytest.mark.parametrize("mean,size", [(1000.0, 1.0), (-3e4, 10.0), (1e-20, 1e-22), (0.0, 1e15)])
def test_data_far_from_zero_or_of_odd_size(mean, size):
    # 1 / sqrt(var + eps) with the variance far below and far above eps too
    x = inputs(2, 24, (40, 40), torch.float32, 3, mean=mean, size=size)
    check_forward(x, 6, rand((24,), 1, mean=1.0, size=0.3), rand((24,), 2), act="none")


def test_one_value_far_from_the_rest():
    # the value a thread measures its differences from
    x = inputs(1, 8, (64, 64), torch.float32, 3).contiguous(memory_format=torch.channels_last)
    x[0, :, 0, 0] = 1e4
    check_forward(x, 2)


def test_constant_groups():
    """Variance zero: h = 0, y = act(b), dx is the rounding of zero times rstd."""
    B = _binding()
    x = torch.full((2, 8, 5, 5), 3.25, device="cuda").contiguous(memory_format=torch.channels_last)
    b = rand((8,), 1)
    y, mean, rstd = B.group_norm_forward(x, 2, None, b, 1e-5, "silu")
    assert (mean == 3.25).all()
    assert ((rstd - 1e-5 ** -0.5).abs() <= 1e-5 ** -0.5 * 4 * U).all()
    want = (b.double() / (1 + torch.exp(-b.double()))).reshape(1, 8, 1, 1)
    assert ((y.double() - want).abs() <= 8 * U * (1 + want.abs())).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_stay_in_their_group(bad):
    B = _binding()
    x = inputs(3, 12, (6, 5), torch.float32, 3).clone(memory_format=torch.preserve_format)
    x[1, 4, 2, 2] = bad
    y, mean, rstd = B.group_norm_forward(x, 3, None, None, 1e-5, "none")
    assert not mean[1, 1].isfinite().item() and y[1, 4:8].isnan().any()
    mean[1, 1], rstd[1, 1] = 0, 0
    assert mean.isfinite().all() and rstd.isfinite().all()
    assert y[0].isfinite().all() and y[2].isfinite().all()
    assert y[1, :4].isfinite().all() and y[1, 8:].isfinite().all()
    dy = inputs(3, 12, (6, 5), torch.float32, 4).clone(memory_format=torch.preserve_format)
    dy[0, 0, 0, 0] = bad
    x[1, 4, 2, 2] = 0.0
    _, mean, rstd = B.group_norm_forward(x, 3)
    dx, _, _ = B.group_norm_backward(dy, x, mean, rstd, 3)
    assert not dx[0, :4].isfinite().all() and dx[0, 4:].isfinite().all() and dx[1:].isfinite().all()


def test_extreme_arguments_of_silu():
    B = _binding()
    x = inputs(1, 2, (50,), torch.float32, 3)
    w = torch.tensor([200.0, 0.0], device="cuda")
    b = torch.tensor([0.0, -120.0], device="cuda")
    y, mean, rstd = B.group_norm_forward(x, 2, w, b, 1e-5, "silu")
    assert y.isfinite().all()
    dx, dw, db = B.group_norm_backward(torch.ones_like(x), x, mean, rstd, 2, w, b, "silu")
    assert dx.isfinite().all() and dw.isfinite().all() and db.isfinite().all()


@pytest.mark.parametrize("act", ("none", "silu"))
@pytest.mark.parametrize("size", [(2, 16, 4, (8, 8)), (1, 30, 6, (7, 5)), (2, 64, 32, (40, 40))])
def test_gradients_against_differences(size, act):
    """(L(p + t v) - L(p - t v)) / 2t for L = sum y dy, in each of x, weight and bias."""
    B = _binding()
    n, c, groups, pos = size
    p = {"x": inputs(n, c, pos, torch.float32, 1), "w": rand((c,), 2, mean=1.0, size=0.3), "b": rand((c,), 3)}
    dy = inputs(n, c, pos, torch.float32, 4)
    _, mean, rstd = B.group_norm_forward(p["x"], groups, p["w"], p["b"], 1e-5, act)
    grads = dict(zip("xwb", B.group_norm_backward(dy, p["x"], mean, rstd, groups, p["w"], p["b"], act)))

    def loss(q):
        y = B.group_norm_forward(q["x"], groups, q["w"], q["b"], 1e-5, act)[0]
        return (y.double() * dy.double()).sum().item()

    t = 2.0 ** -8
    for k in "xwb":
        v = torch.sign(grads[k]) + (grads[k] == 0)  # along the gradient: no cancellation in the sum
        want = (grads[k].double() * v.double()).sum().item()
        up, down = dict(p), dict(p)
        up[k], down[k] = p[k] + t * v, p[k] - t * v
        got = (loss(up) - loss(down)) / (2 * t)
        # third derivatives of the loss along v times t^2 / 6; fp32 rounding of y divided by t
        scale = dy.double().abs().sum().item()
        assert abs(got - want) <= 30 * t * t * (abs(want) + scale) + 40 * U * scale / t


def test_refusals():
    B = _binding()
    x = inputs(2, 12, (4, 4), torch.float32, 1)
    w = torch.ones(12, device="cuda")
    for call in (lambda: B.group_norm_forward(x, 5), lambda: B.group_norm_forward(x, 0),
                 lambda: B.group_norm_forward(x, -3), lambda: B.group_norm_forward(x, 3, eps=-1.0),
                 lambda: B.group_norm_forward(x, 3, eps=math.nan),
                 lambda: B.group_norm_forward(x[:, :, :0], 3)):
        with pytest.raises(B.EfcpError) as ei:
            call()
        assert ei.value.code == B.EINVAL
    for call in (lambda: B.group_norm_forward(x, 3, act="gelu"),
                 lambda: B.group_norm_forward(x.double(), 3), lambda: B.group_norm_forward(x.cpu(), 3),
                 lambda: B.group_norm_forward(x[0, :, 0, 0], 3), lambda: B.group_norm_forward(x, 3, w[:5]),
                 lambda: B.group_norm_forward(x, 3, w.double()), lambda: B.group_norm_forward(x, 3, w.cpu()),
                 lambda: B.group_norm_forward(x, 3, w, w.bfloat16()),
                 lambda: B.group_norm_forward(x, 3, torch.ones(24, device="cuda")[::2])):
        with pytest.raises(ValueError):
            call()
    y, mean, rstd = B.group_norm_forward(x, 3, w)
    for call in (lambda: B.group_norm_backward(y[:1], x, mean, rstd, 3, w),
                 lambda: B.group_norm_backward(y.bfloat16(), x, mean, rstd, 3, w),
                 lambda: B.group_norm_backward(y, x, mean[:1], rstd, 3, w),
                 lambda: B.group_norm_backward(y, x, mean, rstd.double(), 3, w)):
        with pytest.raises(ValueError):
            call()


def test_no_samples():
    B = _binding()
    x = torch.empty((0, 12, 4, 4), device="cuda")
    w = torch.ones(12, device="cuda")
    y, mean, rstd = B.group_norm_forward(x, 3, w, w)
    assert y.shape == x.shape and mean.shape == (0, 3)
    dx, dw, db = B.group_norm_backward(x, x, mean, rstd, 3, w, w)
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all()


def test_autograd_module():
    from paper_2306_06098_b200.norm import GroupNorm, group_norm
    torch.manual_seed(0)
    for act in ("none", "silu"):
        ours = GroupNorm(4, 16, act=act, device="cuda")
        plain = torch.nn.GroupNorm(4, 16, device="cuda", dtype=torch.float64)
        with torch.no_grad():
            ours.weight.copy_(rand((16,), 1, mean=1.0, size=0.3))
            ours.bias.copy_(rand((16,), 2))
            plain.weight.copy_(ours.weight)
            plain.bias.copy_(ours.bias)
        x = inputs(3, 16, (6, 7), torch.float32, 5).detach().requires_grad_(True)
        x64 = x.detach().double().requires_grad_(True)
        dy = inputs(3, 16, (6, 7), torch.float32, 6)
        y = ours(x)
        y.backward(dy)
        y64 = plain(x64)
        y64 = y64 * torch.sigmoid(y64) if act == "silu" else y64
        y64.backward(dy.double())
        for got, ref in ((y, y64), (x.grad, x64.grad), (ours.weight.grad, plain.weight.grad),
                         (ours.bias.grad, plain.bias.grad)):
            assert (got.double() - ref).norm() <= 100 * U * ref.norm()
    x = inputs(2, 6, (3, 3), torch.bfloat16, 7).requires_grad_(True)
    group_norm(x, 2).sum().backward()  # without parameters; dy is broadcast
    assert x.grad.dtype == torch.bfloat16
    with pytest.raises(ValueError):
        GroupNorm(5, 16)
    with pytest.raises(ValueError):
        GroupNorm(4, 16, act="gelu")


def test_another_stream_and_a_captured_graph():
    B = _binding()
    x, dy = inputs(4, 32, (20, 20), torch.float32, 1), inputs(4, 32, (20, 20), torch.float32, 2)
    w, b = rand((32,), 3), rand((32,), 4)
    want = B.group_norm_forward(x, 8, w, b, 1e-5, "silu")
    wantg = B.group_norm_backward(dy, x, want[1], want[2], 8, w, b, "silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.group_norm_forward(x, 8, w, b, 1e-5, "silu", stream=side)
    gotg = B.group_norm_backward(dy, x, got[1], got[2], 8, w, b, "silu", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip((*want, *wantg), (*got, *gotg)):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, mean, rstd = B.group_norm_forward(x, 8, w, b, 1e-5, "silu")
        grads = B.group_norm_backward(dy, x, mean, rstd, 8, w, b, "silu")
    x.copy_(inputs(4, 32, (20, 20), torch.float32, 9))
    graph.replay()
    fresh = B.group_norm_forward(x, 8, w, b, 1e-5, "silu")
    freshg = B.group_norm_backward(dy, x, fresh[1], fresh[2], 8, w, b, "silu")
    for p, q in zip((y, mean, rstd, *grads), (*fresh, *freshg)):
        assert torch.equal(p, q)
