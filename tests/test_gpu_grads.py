"""Norm, clipping and gather of lists of gradients against 64-bit formulas."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # unit roundoff of fp32
# rounding to a type: half its spacing above 1
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
# smallest step between values (of fp16 below its normal range too)
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
# N: per-access sums of at most 8 fp32 products of relative error 8 U, then fp64; halved by the
# root, plus the rounding of the result
NORM_TOL = 6 * U
# f g: the norm's sums, f rounded to fp32, the product rounded to fp32
FACTOR_TOL = 8 * U


def _binding():
    from paper_2306_06098_b200 import binding
    return binding


def values(shape, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def norm64(tensors):
    return math.sqrt(sum(t.double().square().sum().item() for t in tensors
                         if isinstance(t, torch.Tensor) and t.numel()))


def flat64(tensors):
    return torch.cat([torch.zeros(t, dtype=torch.float64, device="cuda") if isinstance(t, int)
                      else t.double().contiguous().reshape(-1) for t in tensors])


def close(got, want, dtype, tol):
    err = (got.double() - want).abs()
    bound = want.abs() * (tol + HALF_ULP[dtype] * (dtype != torch.float32)) + TINY[dtype]
    return bool((err <= bound).all())


def at_odd_address(n, dtype, seed, skip):
    return values(n + skip, dtype, seed)[skip:]


LISTS = {
    "one_value": lambda: [values((1,), torch.float32, 1)],
    "one_of_each_type": lambda: [values((3, 5), t, i) for i, t in enumerate(HALF_ULP)],
    "lengths_around_a_chunk": lambda: [values((n,), t, n) for t in HALF_ULP
                                       for n in (1, 7, 31, 255, 4095, 4096, 4097, 8191, 8193, 16385)],
    "odd_addresses": lambda: [at_odd_address(n, t, n, s) for t in HALF_ULP
                              for s in (1, 2, 3, 5, 7) for n in (1, 2, 9, 4099, 20001)],
    "channels_last": lambda: [values((16, 9, 3, 3), t, 3).contiguous(memory_format=torch.channels_last)
                              for t in HALF_ULP],
    "permuted": lambda: [values((37, 50), torch.float32, 4).t(),
                         values((70, 3, 129), torch.bfloat16, 5).permute(2, 0, 1),
                         values((70, 130, 3), torch.float16, 5).permute(1, 0, 2),
                         values((5, 6, 7, 8), torch.float16, 6).permute(3, 1, 0, 2)],
    "slices": lambda: [values((40, 60), torch.float32, 7)[::2, 1::3],
                       values((40, 60), torch.bfloat16, 8)[:, 5:17],
                       values((6, 7, 8, 9), torch.float16, 9)[1:5, ::2, 1:, ::3]],
    "wide_transposes": lambda: [values((65, 4097), torch.float32, 21).t(),
                                values((4097, 65), torch.bfloat16, 22).t(),
                                values((2, 100_001), torch.float16, 23).t(),
                                values((100_001, 2), torch.float32, 24).t()],
    "rank_zero_and_ones": lambda: [values((), torch.float32, 10), values((1, 1, 4, 1), torch.bfloat16, 11),
                                   values((4, 1, 3), torch.float32, 12).transpose(0, 2)],
    "many_tensors": lambda: [values((1 + i % 97,), list(HALF_ULP)[i % 3], i) for i in range(1500)],
    "many_strided": lambda: [values((3 + i % 5, 4 + i % 7), torch.float32, i).t() for i in range(700)],
    "empty_ones": lambda: [values((0,), torch.float32, 1), values((0, 3), torch.bfloat16, 1).t(),
                           values((5,), torch.float32, 2)],
    "large": lambda: [values((1024, 2049), torch.float32, 30), values((8_000_003,), torch.bfloat16, 31)],
}


@pytest.mark.parametrize("name", LISTS)
def test_norm(name):
    B = _binding()
    ts = LISTS[name]()
    want = norm64(ts)
    got = B.grad_norm(ts)
    assert got.dtype == torch.float32 and got.shape == ()
    assert abs(got.item() - want) <= NORM_TOL * want
    assert B.grad_norm(tuple(ts), scale=0.125).item() == got.item() * 0.125
    out = torch.zeros((), device="cuda")
    assert B.grad_norm(ts, out=out) is out and out.item() == got.item()  # repeats bit for bit


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("ratio,scale", [(0.3, 1.0), (0.7, 1.0 / 1024), (2.0, 0.25)])
def test_clip(name, ratio, scale):
    B = _binding()
    ts = LISTS[name]()
    before = [t.clone() for t in ts]
    norm = norm64(ts) * scale
    got = B.clip_grads(ts, ratio * norm, scale=scale)
    assert abs(got.item() - norm) <= NORM_TOL * norm
    f = scale * min(1.0, ratio)
    for t, b in zip(ts, before):
        assert close(t, b.double() * f, t.dtype, FACTOR_TOL)


def test_clip_writes_nothing_when_there_is_nothing_to_do():
    B = _binding()
    ts = [values((513,), t, i) for i, t in enumerate(HALF_ULP)]
    ts[0][7] = -0.0
    before = [t.clone() for t in ts]
    B.clip_grads(ts, 1e9)
    B.clip_grads(ts, math.inf)
    for t, b in zip(ts, before):
        assert torch.equal(t.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("max_ratio,scale,norm", [(0.0, 1.0, False), (0.0, 0.5, True),
                                                   (0.4, 1.0, True), (3.0, 1.0 / 1024, False)])
def test_gather(name, max_ratio, scale, norm):
    B = _binding()
    ts = LISTS[name]()
    ts = ts[:1] + [5] + ts[1:] + [1, 4099]  # parameters without a gradient
    want = flat64(ts)
    n64 = norm64(ts) * scale
    before = [t.clone() for t in ts if isinstance(t, torch.Tensor)]
    for skip in (0, 1, 3):  # the flat vector at odd addresses, with guards around it
        buf = torch.full((want.numel() + skip + 5,), -7.0, device="cuda")
        flat = buf[skip:skip + want.numel()]
        got = B.gather_grads(ts, flat, max_norm=max_ratio * n64, scale=scale, norm=norm)
        assert (got is None) == (not norm)
        if norm:
            assert abs(got.item() - n64) <= NORM_TOL * n64
        f = scale * (min(1.0, max_ratio) if max_ratio else 1.0)
        assert close(flat, want * f, torch.float32, FACTOR_TOL)
        if f == 1.0 or f == 0.5:  # exact factors: exact products
            assert torch.equal(flat.double(), want * f)
        assert (buf[:skip] == -7).all() and (buf[skip + want.numel():] == -7).all()
    for t, b in zip([t for t in ts if isinstance(t, torch.Tensor)], before):
        assert torch.equal(t, b)


def test_gather_copies_bits():
    B = _binding()
    a = torch.randint(-2 ** 31, 2 ** 31 - 1, (10_007,), dtype=torch.int32, device="cuda")
    a = a.view(torch.float32)  # every kind of value, NaN payloads among them
    for t in (a, a[1:], a[:10_000].view(100, 100).t()):
        flat = torch.empty(t.numel(), device="cuda")
        B.gather_grads([t], flat)
        assert torch.equal(flat.view(torch.int32), t.contiguous().view(-1).view(torch.int32))


def test_gradients_of_broadcast_inputs():
    B = _binding()
    one = values((1,), torch.float32, 1)
    row = values((1, 50), torch.bfloat16, 2)
    ts = [one.expand(1000), row.expand(30, 50), values((7, 1), torch.float32, 3).expand(7, 9)]
    want = flat64(ts)
    flat = torch.empty(want.numel(), device="cuda")
    norm = B.gather_grads(ts, flat, norm=True)
    assert torch.equal(flat.double(), want)
    assert abs(norm.item() - norm64(ts)) <= NORM_TOL * norm64(ts)
    assert abs(B.grad_norm(ts).item() - norm64(ts)) <= NORM_TOL * norm64(ts)
    for t in ts:  # elements share memory: cannot be scaled in place
        with pytest.raises(B.EfcpError) as ei:
            B.clip_grads([t], 1e-3)
        assert ei.value.code == B.EINVAL


@pytest.mark.parametrize("size", [1e30, 3e-30, 1e-40])
def test_squares_that_leave_the_range_of_fp32(size):
    B = _binding()
    t = (torch.randn(30_000, dtype=torch.float64) * size).float().cuda()
    want = norm64([t])
    assert abs(B.grad_norm([t]).item() - want) <= NORM_TOL * want + 2.0 ** -149
    mixed = [t, torch.zeros(5000, device="cuda"), values((10,), torch.float32, 1)]
    want = norm64(mixed)
    assert abs(B.grad_norm(mixed).item() - want) <= NORM_TOL * want
    if size > 1:
        c = t.clone()
        B.clip_grads([c], 1.0)
        assert close(c, t.double() / norm64([t]), torch.float32, FACTOR_TOL)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(bad):
    B = _binding()
    ts = [values((100,), torch.float32, 1), values((5000,), torch.bfloat16, 2)]
    ts[1][4321] = bad
    before = [t.clone() for t in ts]
    norm = B.clip_grads(ts, 1.0)
    assert not math.isfinite(norm.item())
    for t, b in zip(ts, before):  # nothing is clipped
        assert torch.equal(t.view(torch.int16), b.view(torch.int16))
    flat = torch.empty(5100, device="cuda")
    norm = B.gather_grads(ts, flat, max_norm=1.0, norm=True)
    assert not math.isfinite(norm.item())
    assert torch.equal(flat, flat64(before).float()) or math.isnan(bad)
    assert not math.isfinite(flat[100 + 4321].item())
    assert B.grad_norm(before[:1]).isfinite().item()  # nothing is left behind in the workspace


def test_empty_lists():
    B = _binding()
    assert B.grad_norm([]).item() == 0.0
    assert B.grad_norm([torch.empty(0, device="cuda")]).item() == 0.0
    assert B.clip_grads([], 1.0).item() == 0.0
    assert B.gather_grads([], torch.empty(0, device="cuda"), norm=True).item() == 0.0
    flat = torch.full((12,), 3.0, device="cuda")
    assert B.gather_grads([5, 7], flat, max_norm=1.0, norm=True).item() == 0.0
    assert (flat == 0).all()
    z = [torch.zeros(100, device="cuda")]
    assert B.clip_grads(z, 1.0).item() == 0.0 and (z[0] == 0).all()


def test_refusals():
    B = _binding()
    t = values((10, 10), torch.float32, 1)
    for call in (lambda: B.clip_grads([t], 0.0), lambda: B.clip_grads([t], -1.0),
                 lambda: B.clip_grads([t], math.nan), lambda: B.grad_norm([t], scale=0.0),
                 lambda: B.grad_norm([t], scale=math.inf),
                 lambda: B.gather_grads([t], torch.empty(99, device="cuda")),
                 lambda: B.gather_grads([t, -1], torch.empty(99, device="cuda")),
                 lambda: B.gather_grads([t], torch.empty(100, device="cuda"), max_norm=-1.0)):
        with pytest.raises(B.EfcpError) as ei:
            call()
        assert ei.value.code == B.EINVAL
    deep = values((3, 3, 3, 3, 3, 3), torch.float32, 1)[:2, :2, :2, :2, :2, :2]
    with pytest.raises(B.EfcpError):  # five dimensions that do not merge
        B.grad_norm([deep])
    for bad in ([t.cpu()], [t.double()], [t.int()], [t.to_sparse()], [None], ["x"], [3]):
        with pytest.raises((ValueError, TypeError)):
            B.grad_norm(bad, out=torch.zeros((), device="cuda"))
    with pytest.raises(TypeError):
        B.grad_norm(iter([t]), out=torch.zeros((), device="cuda"))
    with pytest.raises(ValueError):
        B.gather_grads([t], torch.empty(100, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.gather_grads([t], torch.empty(200, device="cuda")[::2])
    assert torch.equal(t, values((10, 10), torch.float32, 1))


def test_another_stream_and_a_captured_graph():
    B = _binding()
    ts = [values((300, 301), torch.float32, 1), values((777,), torch.bfloat16, 2)]
    d = sum(t.numel() for t in ts)
    flat = torch.empty(d, device="cuda")
    want = flat64(ts)
    n64 = norm64(ts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm = B.gather_grads(ts, flat, max_norm=0.5 * n64, norm=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert close(flat, want * 0.5, torch.float32, FACTOR_TOL)
    assert abs(norm.item() - n64) <= NORM_TOL * n64
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = B.gather_grads(ts, flat, max_norm=0.5 * n64, norm=True)
    for k in (1, 2, 3):
        flat.zero_()
        graph.replay()
        assert abs(norm.item() - n64 * 2.0 ** (k - 1)) <= NORM_TOL * n64 * 2.0 ** (k - 1)
        assert close(flat, want * 0.5, torch.float32, FACTOR_TOL)
        for t in ts:
            t.mul_(2.0)


def test_clipping_is_an_in_place_change_for_autograd():
    B = _binding()
    t = values((100,), torch.float32, 1)
    version = t._version
    B.grad_norm([t])
    assert t._version == version
    B.clip_grads([t], 1e-3)
    assert t._version == version + 1


def test_values_of_numpy_agree():
    """The whole call against numpy in 64 bits, on the layout of a small convolutional model."""
    B = _binding()
    rng = np.random.default_rng(3)
    host = [rng.standard_normal(s).astype(np.float32) for s in ((16, 3, 3, 3), (16,), (32, 16, 3, 3), (10, 64))]
    dev = [torch.from_numpy(h).cuda() for h in host]
    dev = [t.contiguous(memory_format=torch.channels_last) if t.dim() == 4 else t for t in dev]
    norm = math.sqrt(sum((h.astype(np.float64) ** 2).sum() for h in host))
    flat = torch.empty(sum(h.size for h in host), device="cuda")
    got = B.gather_grads(dev, flat, max_norm=2.0, norm=True)
    want = np.concatenate([h.astype(np.float64).reshape(-1) for h in host]) * (2.0 / norm)
    assert abs(got.item() - norm) <= NORM_TOL * norm
    assert np.all(np.abs(flat.cpu().numpy() - want) <= FACTOR_TOL * np.abs(want))
