"""Tensors that share memory in a list to be clipped: refused before anything is enqueued, through the C ABI and
without a GPU; tensors whose elements lie between each other's are not."""
import itertools
import random

import pytest
import torch

from paper_2306_06098_b200 import binding as B

FAKE = 0x7F0000000000  # never read: there is no device

no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")


def describe(t):
    """A descriptor of the layout of a tensor, at a made-up address."""
    d = B.TensorDesc(data=FAKE + t.storage_offset() * t.element_size(), numel=t.numel(), dtype=B.DTYPES[t.dtype])
    if not t.is_contiguous():
        d.rank = t.dim()
        for k in range(t.dim()):
            d.size[k], d.stride[k] = t.size(k), t.stride(k)
    return d


def clip(*ts):
    return B._lib.efcp_grads_clip((B.TensorDesc * len(ts))(*map(describe, ts)), len(ts), 1.0, 1.0, FAKE, FAKE, None)


def bytes_of(t):
    w = t.element_size()
    return {w * (t.storage_offset() + sum(i * s for i, s in zip(ix, t.stride()))) + k
            for ix in itertools.product(*map(range, t.shape)) for k in range(w)}


@no_device
def test_the_same_elements_twice():
    g = torch.zeros(40)
    m = torch.zeros(6, 8)
    for ts in ((g, g), (g, g[:10]), (g[5:], g[:6]), (g[:20], torch.zeros(3), g[19:]), (m, m[2:4, 3:5]), (m[:, :5], m[:, 4:]),
               (m.t(), m[0]), (m[::2], m[2]), (m[1:4, 2:6], m[3:5, 5:8]), (g[39:], g)):
        assert clip(*ts) == B.EINVAL
        assert clip(*reversed(ts)) == B.EINVAL


@no_device
def test_neighbours_are_accepted():
    g = torch.zeros(4000)
    m = torch.zeros(60, 80)
    c = torch.zeros(4, 5, 6, 7)
    for ts in ((g[:10], g[10:]), (g[3:10], g[10:11], g[:3]), (m[:, :50], m[:, 50:]), (m[::2], m[1::2]), (m[:30], m[30:]),
               (m[:, ::3], m[:, 1::3], m[:, 2::3]), (m.t()[:20], m.t()[20:]), (m[:, :40], m[:30, 40:], m[30:, 40:]),
               (c[:, :2], c[:, 2:]), (c[..., 0], c[..., 1:]), (c[:, :, :3, ::2], c[:, :, :3, 1::2], c[:, :, 3:]),
               tuple(m[:, k] for k in range(80)), (g[:0], g), (g, g[:0])):
        assert clip(*ts) == B.ECUDA  # gets as far as asking for the device
        assert clip(*reversed(ts)) == B.ECUDA


@no_device
def test_two_types_in_one_buffer():
    wide = torch.zeros(30)
    half = torch.zeros(60, dtype=torch.bfloat16)  # the same made-up bytes
    assert clip(wide[:15], half[30:]) == B.ECUDA
    assert clip(wide[:15], half[29:]) == B.EINVAL
    assert clip(wide[15:], half[:30]) == B.ECUDA
    assert clip(wide[15:], half[:31]) == B.EINVAL


@no_device
@pytest.mark.parametrize("seed", range(8))
def test_pairs_of_slices_against_their_elements(seed):
    rng = random.Random(seed)
    kinds = [0, 0]
    for _ in range(400):
        base = torch.zeros([rng.randint(1, 6) for _ in range(rng.randint(1, 4))])
        pair = []
        for _ in range(2):
            t = base
            for k in range(t.dim()):
                a = rng.randrange(t.size(k))
                t = t.narrow(k, a, rng.randint(1, t.size(k) - a))
                ix = [slice(None)] * t.dim()
                ix[k] = slice(None, None, rng.choice((1, 1, 2, 3)))
                t = t[tuple(ix)]
            order = list(range(t.dim()))
            rng.shuffle(order)
            pair.append(t.permute(order))
        share = bool(bytes_of(pair[0]) & bytes_of(pair[1]))
        kinds[share] += 1
        assert clip(*pair) == (B.EINVAL if share else B.ECUDA), [(t.storage_offset(), t.shape, t.stride()) for t in pair]
    assert min(kinds) >= 20


@no_device
def test_unlike_strides():
    """Two layouts of one buffer that have nothing in common."""
    g = torch.zeros(1000)
    for a, b in ((g.as_strided((7, 9), (90, 10), 0), g.as_strided((5, 4), (70, 10), 3)),
                 (g.as_strided((30,), (15,), 0), g.as_strided((20,), (21,), 1)),
                 (g.as_strided((10,), (2,), 0), g.as_strided((10, 5), (20, 2), 1))):
        share = bool(bytes_of(a) & bytes_of(b))
        assert clip(a, b) == clip(b, a) == (B.EINVAL if share else B.ECUDA)


@no_device
def test_extents_beyond_the_address_space_are_refused():
    d = B.TensorDesc(data=FAKE, numel=100, dtype=0, rank=2)
    d.size[0], d.size[1], d.stride[0], d.stride[1] = 10, 10, 1 << 62, 1
    one = (B.TensorDesc * 1)(d)
    assert B._lib.efcp_grads_clip(one, 1, 1.0, 1.0, FAKE, FAKE, None) == B.EINVAL
    assert B._lib.efcp_grads_norm(one, 1, 1.0, FAKE, FAKE, None) == B.EINVAL


@pytest.mark.gpu
def test_on_the_device():
    g = torch.randn(1000, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda")
    before = g.clone()
    for ts in ([g, g], [g, g[:10]], [g.view(10, 100)[:, :50], g.view(10, 100)[:, 49:]]):
        with pytest.raises(B.EfcpError) as ei:
            B.clip_grads(ts, 1.0)
        assert ei.value.code == B.EINVAL
        assert torch.equal(g, before)
    m = g.view(10, 100)
    norm = B.clip_grads([m[:, :37], m[:, 37:]], 1.0)
    n64 = before.double().norm().item()
    assert abs(norm.item() - n64) <= 6 * 2.0 ** -24 * n64
    want = before.double() / n64
    assert ((g.double() - want).abs() <= 8 * 2.0 ** -24 * want.abs()).all()
