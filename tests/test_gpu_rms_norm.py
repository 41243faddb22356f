"""RMS norm of a residual stream (with dropout, and with an output in 8 bits) against 64-bit formulas."""
import itertools

import pytest
import torch

from philox import kept, threshold

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = (torch.float32, torch.bfloat16, torch.float16)
EPS = 1e-6
RNG = (0x1234567890ABCDEF, 77)


def B():
    from paper_2306_06098_b200 import binding
    return binding


def rand(shape, seed, dtype=torch.float32, pad=0, shift=0):
    """Rows of a wider tensor (pad), that start `shift` elements off."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn(*shape[:-1], shape[-1] + pad + shift, device="cuda", generator=g).to(dtype)
    return wide[..., shift:shift + shape[-1]]


def sum64(x, residual, p, rng):
    """h before its rounding."""
    s = x.double()
    if p:
        s = torch.where(kept(x.shape, p, *rng).cuda(), s * (65536 / (65536 - threshold(p))), 0.0)
    return s if residual is None else s + residual.double()


def check_forward(x, residual=None, weight=None, p=0.0, eps=EPS):
    y, h, rstd = B().rms_norm_forward(x, weight, eps, residual, p, RNG)
    assert y.shape == h.shape == x.shape and y.dtype == h.dtype == x.dtype and rstd.shape == x.shape[:-1]
    d = x.shape[-1]
    want_h = sum64(x, residual, p, RNG)
    if residual is None and not p:
        assert h is x or torch.equal(h, x)
    else:
        # the product with the scale and the addition round in fp32, the result to its type
        part = x.double().abs() * (65536 / (65536 - threshold(p))) if p else x.double().abs()
        off = 2 * U * (part + want_h.abs())
        assert ((h.double() - want_h).abs() <= off + HALF[x.dtype] * (want_h.abs() + off) + TINY[x.dtype]).all()
    h64 = h.double()
    r64 = 1 / (h64.square().mean(-1, keepdim=True) + eps).sqrt()
    # squares of eight, chunks of a lane, lanes and warps: fewer than 8 + d / 256 + 5 + 32 roundings of
    # positive terms; half of that in the root, which is within 2 units itself, and the mean's product
    rel = (0.5 * (8 + d / 256 + 5 + 32 + 3) + 3) * U
    assert ((rstd.double() - r64[..., 0]).abs() <= rel * r64[..., 0]).all()
    want = h64 * r64 * (1.0 if weight is None else weight.double())
    bound = (rel + 3 * U) * want.abs()
    assert ((y.double() - want).abs() <= bound + HALF[x.dtype] * (want.abs() + bound) + TINY[x.dtype]).all()
    again = B().rms_norm_forward(x, weight, eps, residual, p, RNG)
    assert all(torch.equal(a, b) for a, b in zip((y, h, rstd), again))
    return y, h, rstd


SIZES = [(1, 1), (1, 7), (3, 8), (5, 31), (2, 256), (7, 257), (1, 4096), (33, 768), (4, 1111), (2, 5000),
         (3, 16384), (2, 16385), (1, 40000), (1, 70001)]


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_sizes(rows, d, dtype):
    x, r, w = rand((rows, d), 1, dtype), rand((rows, d), 2, dtype), rand((d,), 3)
    check_forward(x, None, w)
    check_forward(x, r, w)
    check_forward(x, r, None, 0.1)
    check_forward(x, None, w, 0.5)


@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (8, 8), (64, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_rows_of_a_wider_tensor(pad, shift, dtype):
    for d in (264, 1001):
        x, r = rand((9, d), 1, dtype, pad, shift), rand((9, d), 2, dtype)
        check_forward(x, r, rand((d,), 3), 0.25)
        check_forward(r, x, rand((d,), 3, torch.bfloat16), 0.25)


def test_forward_many_rows_and_shapes():
    check_forward(rand((20000, 24), 1), rand((20000, 24), 2), None, 0.1)
    check_forward(rand((3000, 1024), 1, torch.bfloat16), rand((3000, 1024), 2, torch.bfloat16), rand((1024,), 3))
    x = rand((4, 5, 6, 40), 4)
    check_forward(x.transpose(0, 2), x.permute(2, 1, 0, 3).contiguous(), rand((40,), 3), 0.3)  # copied first
    check_forward(x[:, :, 0], None, None)
    check_forward(rand((300,), 5), None, rand((300,), 6))  # one row without other dimensions
    check_forward(rand((1, 64), 7).expand(5, 64), None, None)
    for shape in ((0, 16), (3, 0, 16)):
        y, h, rstd = B().rms_norm_forward(rand(shape, 1), None)
        assert y.shape == shape and rstd.shape == shape[:-1]


def test_values_that_are_special():
    d = 512
    x = rand((6, d), 1)
    x[0] = 0
    x[1] *= 1e18
    x[2] *= 1e-20
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    y, _, rstd = B().rms_norm_forward(x, None, EPS)
    assert (y[0] == 0).all() and rstd[0].item() == pytest.approx(1e3, rel=1e-6)
    check_forward(x[1:3])
    check_forward(x[5:])
    assert rstd[3].item() == 0 and y[3, 5].isnan() and (y[3, :5] == 0).all()
    assert y[4].isnan().all() and not y[5].isnan().any()
    # what is dropped is gone, whatever it was
    keep = kept((1, d), 0.5, *RNG).cuda()
    bad = torch.where(keep, x[5:], torch.tensor(float("nan"), device="cuda"))
    a, b = B().rms_norm_forward(bad, None, EPS, None, 0.5, RNG), B().rms_norm_forward(x[5:], None, EPS, None, 0.5, RNG)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ backward
def check_backward(rows, d, dtype, weight=None, with_dh=True, p=0.0, pad=0, want=(True, True, True)):
    h, dy = rand((rows, d), 1, dtype, pad), rand((rows, d), 2, dtype)
    dh = rand((rows, d), 3, dtype) if with_dh else None
    rstd = (1 / (h.double().square().mean(-1) + EPS).sqrt()).float()
    got = B().rms_norm_backward(dy, h, rstd, weight, dh, p, RNG, want)
    w = torch.ones(d, dtype=torch.float64, device="cuda") if weight is None else weight.double()
    h64, dy64, r = h.double(), dy.double(), rstd.double()[:, None]
    g = dy64 * w
    terms = (g * h64).abs().mean(-1, keepdim=True) * r * r
    dz = r * (g - h64 * r * r * (g * h64).mean(-1, keepdim=True))
    # the row's sum: fewer than 8 + d / 256 + 5 + 32 additions, each term with two products
    off = r * (4 * U * g.abs() + h64.abs() * terms * (8 + d / 256 + 5 + 32 + 8) * U) + 2 * U * dz.abs()
    if with_dh:
        dz = dz + dh.double()
        off = off + U * dz.abs()

    def near(a, b, off):
        assert ((a.double() - b).abs() <= off + HALF[dtype] * (b.abs() + off) + TINY[dtype]).all()

    if want[1]:
        near(got[1], dz, off)
    if want[0]:
        if p:
            keep, s = kept((rows, d), p, *RNG).cuda(), 65536 / (65536 - threshold(p))
            near(got[0], torch.where(keep, dz * s, 0.0), torch.where(keep, off * s + U * dz.abs() * s, 0.0))
        elif want[1]:
            assert got[0] is got[1]
        else:
            near(got[0], dz, off)
    if weight is None or not want[2]:
        assert got[2] is None
    else:
        t = dy64 * h64 * r
        # rows one after another in a slot (at most all of them), then the slots: 32 lanes of them
        n = min(rows, 2 + rows // 100) + 8
        bound = t.abs().sum(0) * (n + 40 + rows / 1000) * U
        want_w = t.sum(0)
        half = 0.0 if weight.dtype == torch.float32 else HALF[weight.dtype]
        assert ((got[2].double() - want_w).abs() <= bound + half * (want_w.abs() + bound) + TINY[weight.dtype]).all()
    for i in range(3):
        assert (got[i] is None) == (not want[i] or (i == 2 and weight is None))
    again = B().rms_norm_backward(dy, h, rstd, weight, dh, p, RNG, want)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("rows,d", SIZES + [(5000, 40), (700, 2304)])
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_sizes(rows, d, dtype):
    check_backward(rows, d, dtype, rand((d,), 9))
    check_backward(rows, d, dtype, rand((d,), 9, dtype), with_dh=False, p=0.3)
    check_backward(rows, d, dtype, None, p=0.1, pad=3)


@pytest.mark.parametrize("want", list(itertools.product((False, True), repeat=3)))
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_backward_of_what_is_wanted(want, p):
    check_backward(37, 520, torch.float32, rand((520,), 9), p=p, want=want)
    check_backward(2, 17000, torch.bfloat16, rand((17000,), 9), p=p, want=want)


def test_backward_without_rows():
    e = torch.empty(0, 8, device="cuda")
    dx, dr, dw = B().rms_norm_backward(e, e, torch.empty(0, device="cuda"), torch.ones(8, device="cuda"))
    assert dx.shape == (0, 8) and (dw == 0).all()


# ------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (4, 256), (7, 2048), (5, 1111), (2, 16400), (300, 520)])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize(rows, d, block, format, dtype):
    x, r, w = rand((rows, d), 1, dtype), rand((rows, d), 2, dtype), rand((d,), 3)
    x[0, :] = 0
    r[0, : d // 2] = 0  # blocks of zeros
    q, scales, h = B().rms_norm_quantize(x, w, EPS, r, block, format)
    assert q.dtype == (torch.float8_e4m3fn if format == "e4m3" else torch.int8) and q.shape == x.shape
    assert torch.equal(h, (x.float() + r.float()).to(dtype))
    h64 = h.double()
    z = h64 / (h64.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    wide = block or d
    blocks = -(-d // wide)
    assert scales.shape == (rows, blocks)
    most = 448.0 if format == "e4m3" else 127.0
    rel = (0.5 * (8 + d / 256 + 5 + 32 + 3) + 8) * U
    for k in range(blocks):
        part, qk, s = z[:, k * wide:(k + 1) * wide], q[:, k * wide:(k + 1) * wide], scales[:, k].double()
        top = part.abs().amax(1)
        assert torch.where(top > 0, (s - top / most).abs() <= rel * top / most, s == 1).all()
        value = qk.double() * s[:, None]
        # half a step: of 2^-3 relative and 2^-9 at least (e4m3), of 1 (int8)
        step = (part.abs() * 2.0 ** -4).maximum(s[:, None] * 2.0 ** -10) if format == "e4m3" else 0.5 * s[:, None]
        assert ((value - part).abs() <= step * (1 + 2.0 ** -10) + 4 * rel * part.abs()).all()


def test_quantize_bad_values():
    x = rand((3, 256), 1)
    x[0, 3], x[1, 200] = float("nan"), float("inf")
    for block in (0, 64):
        q, s, _ = B().rms_norm_quantize(x, None, EPS, None, block)
        assert s[0].isnan().all() and (q[0].float() == 0).all()  # NaN in the row's sum
        assert s[1].isnan().any() and not s[2].isnan().any()
        back = q.float() * s.repeat_interleave(256 // s.shape[1], dim=1)
        assert back[0].isnan().all() and back[1, 200].isnan()


# ------------------------------------------------------------------ autograd, streams, graphs
@pytest.mark.parametrize("dtype", TYPES)
def test_autograd(dtype):
    from paper_2306_06098_b200 import norm
    x, r, w = rand((6, 5, 48), 1, dtype), rand((6, 5, 48), 2, dtype), rand((48,), 3)
    cy, ch = rand(x.shape, 4, dtype), rand(x.shape, 5, dtype)
    for leaf in (x, r, w):
        leaf.requires_grad_(True)
    y, h = norm.add_rms_norm(x, r, w, EPS, 0.25, RNG)
    got = torch.autograd.grad((y, h), (x, r, w), (cy, ch))
    # the same with the rounded h in 64 bits
    keep, s = kept(x.shape, 0.25, *RNG).cuda(), 65536 / (65536 - threshold(0.25))
    h64 = h.detach().double().requires_grad_(True)
    w64 = w.detach().double().requires_grad_(True)
    y64 = h64 / (h64.square().mean(-1, keepdim=True) + EPS).sqrt() * w64
    dh64, dw64 = torch.autograd.grad((y64 * cy.double()).sum() + (h64 * ch.double()).sum(), (h64, w64))
    for a, b in zip(got, (torch.where(keep, dh64 * s, 0.0), dh64, dw64)):
        assert ((a.double() - b).abs() <= 2 * HALF[dtype] * b.abs() + 200 * U * 10).all()
    only_h = torch.autograd.grad(norm.add_rms_norm(x, r, w, EPS, 0.25, RNG)[1], (x, r), ch)
    assert torch.equal(only_h[1], ch)
    assert norm.rms_norm(x, None).shape == x.shape


def test_gradient_against_differences():
    from paper_2306_06098_b200 import norm
    x, w, c = rand((3, 20), 1).requires_grad_(True), rand((20,), 2).requires_grad_(True), rand((3, 20), 3)
    gx, gw = torch.autograd.grad((norm.rms_norm(x, w, EPS) * c).sum(), (x, w))
    step = 2.0 ** -7

    def f(x, w):
        return (norm.rms_norm(x, w, EPS).double() * c.double()).sum().item()

    with torch.no_grad():
        for i in range(0, 60, 7):
            e = torch.zeros(60, device="cuda")
            e[i] = step
            e = e.view(3, 20)
            slope = (f(x + e, w) - f(x - e, w)) / (2 * step)
            # third derivatives of order 10 times step^2 / 6, and the rounding of 60 values over the step
            assert abs(slope - gx.view(-1)[i].item()) < 10 * step ** 2 + 60 * 16 * U / step
        for i in range(0, 20, 3):
            e = torch.zeros(20, device="cuda")
            e[i] = step
            slope = (f(x, w + e) - f(x, w - e)) / (2 * step)
            assert abs(slope - gw[i].item()) < 60 * 16 * U / step


def test_module_in_a_graph_draws_new_masks():
    from paper_2306_06098_b200 import norm
    m = norm.RMSNorm(64, p=0.5, seed=5, device="cuda")
    x, r = rand((4, 64), 1), torch.zeros(4, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m(x, r)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, h = m(x, r)
    seen = []
    for k in range(3):
        g.replay()
        seen.append(h.clone())
        assert torch.equal(h != 0, kept((4, 64), 0.5, 5, 1 + k).cuda())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])
    m.eval()
    assert torch.equal(m(x, r)[1], x)
    with pytest.raises(ValueError):
        m(rand((4, 32), 1))


def test_another_stream():
    x, r = rand((500, 768), 1, torch.bfloat16), rand((500, 768), 2, torch.bfloat16)
    want = B().rms_norm_forward(x, None, EPS, r, 0.1, RNG)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B().rms_norm_forward(x, None, EPS, r, 0.1, RNG, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_offsets_beyond_32_bits():
    rows, d = 3, 1000
    big = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (rows, d), (2 ** 30, 1))
    x.copy_(rand((rows, d), 1, torch.bfloat16))
    check_forward(x, rand((rows, d), 2, torch.bfloat16), rand((d,), 3), 0.1)


# ------------------------------------------------------------------ many rows, begun anywhere
ODD = [(300, 1), (299, 7), (1000, 33), (301, 127), (600, 250), (1531, 1111), (297, 2051), (310, 4099), (298, 8179)]


@pytest.mark.parametrize("rows,d", ODD)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_odd_rows(rows, d, dtype):
    x, r, w = rand((rows, d), 1, dtype), rand((rows, d), 2, dtype), rand((d,), 3)
    check_forward(x, r, w, 0.1)
    check_forward(x, None, w)
    check_backward(rows, d, dtype, w)
    check_backward(rows, d, dtype, rand((d,), 9, dtype), with_dh=False, p=0.3, pad=1)


@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 3), (2, 1), (5, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_odd_rows_of_wider_tensors(pad, shift, dtype):
    for rows, d in ((299, 45), (320, 1001), (300, 264)):
        x, r = rand((rows, d), 1, dtype, pad, shift), rand((rows, d), 2, dtype, shift)
        check_forward(x, r, rand((d,), 3, torch.bfloat16), 0.25)
        check_forward(r, x, None)
        check_backward(rows, d, dtype, rand((d,), 9), pad=pad)
    check_forward(rand((1, 1001), 7, dtype).expand(400, 1001), rand((400, 1001), 8, dtype), None)


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_quantize_many_rows(format, dtype):
    for rows, d, block in ((300, 1111, 0), (297, 77, 0), (400, 40, 32), (300, 1000, 64), (350, 4104, 128), (300, 96, 0), (9600, 8, 32),
                          (9600, 16, 64), (9600, 24, 128), (9600, 104, 64), (9600, 128, 128), (9600, 200, 32)):
        test_quantize(rows, d, block, format, dtype)


@pytest.mark.parametrize("rows", [3, 400])
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_quantize_values_whose_scale_is_tiny(rows, format):
    # the inverse of such a scale is beyond fp32
    w = torch.full((64,), 2.0 ** -126, device="cuda")
    x = rand((rows, 64), 1)
    q, s, _ = B().rms_norm_quantize(x, w, EPS, None, 0, format)
    z = x.double() / (x.double().square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    most = 448.0 if format == "e4m3" else 127.0
    tiny, s = 2.0 ** -149, s.double()
    assert s.shape == (rows, 1)
    # subnormal products and scales: half a step of 2^-149 each; the norm's own error as in test_quantize
    rel = (0.5 * (8 + 64 / 256 + 5 + 32 + 3) + 8) * U
    top = z.abs().amax(1, keepdim=True)
    assert ((s - top / most).abs() <= rel * top / most + 2 * tiny).all()
    value = q.double() * s
    step = (z.abs() * 2.0 ** -4).maximum(s * 2.0 ** -10) if format == "e4m3" else 0.5 * s
    assert ((value - z).abs() <= step * (1 + 2.0 ** -10) + 4 * rel * z.abs() + 2 * tiny).all()
