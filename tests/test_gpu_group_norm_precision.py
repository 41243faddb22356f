"""Group norm: how exact the statistics are, against 64 bits, where sums in fp32 are easily spoilt."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def channels_last(n, c, pos, dtype, seed, spread=True):
    """(n, c, *pos), channels last; with `spread` the channels differ in mean and size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, *pos, c), generator=g, device="cuda")
    if spread:
        x.mul_(torch.exp(0.3 * torch.randn(c, generator=g, device="cuda")))
        x.add_(torch.randn(c, generator=g, device="cuda"))
    return x.to(dtype).permute(0, len(pos) + 1, *range(1, len(pos) + 1))


def statistics64(x, groups, eps=1e-5):
    v = x.double().reshape(x.shape[0], groups, -1)
    mean = v.mean(2, keepdim=True)
    var = (v - mean).square().mean(2)
    return mean[..., 0], (var + eps).rsqrt(), var.sqrt()


def statistics(x, groups):
    from paper_2306_06098_b200 import binding
    return binding.group_norm_forward(x, groups)[1:]


# one block a sample, clusters, several tiles, every access width, samples that are streamed
SIZES = [(128, 16, 8, (32, 32)), (2, 1380, 23, (24, 5)), (25, 300, 5, (68, 3)), (43, 58, 2, (3, 2)), (2, 68, 4, (8, 37)),
         (144, 114, 3, (1, 32)), (2, 1036, 28, (101, 61)), (161, 444, 12, (43, 3)), (1, 128, 32, (130, 130)),
         (3, 65, 13, (200, 160)), (64, 64, 32, (56, 56))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_error_of_the_mean(size, dtype):
    n, c, groups, pos = size
    x = channels_last(n, c, pos, dtype, 5)
    mean, _ = statistics(x, groups)
    m64, _, sigma = statistics64(x, groups)
    # rounding the result: U |mean| at most.  A thread's fp32 sum of n <= 64 differences of about
    # sigma: its partial sums grow to n sigma, their roundings together to U sigma sqrt(n) / 3
    # <= 2.7 U sigma, and the independent ones of the group's 16 threads and more average out to
    # less than 0.7 U sigma.  What follows is held in 64 bits.
    err = (mean.double() - m64).square().mean().sqrt().item()
    assert err <= U * (sigma + m64.abs()).square().mean().sqrt().item(), err / U


# groups of one channel (a thread then has a whole column, or a chunk of it, to itself) and larger
# ones; resident and streamed
FIRST = [(3, 127, 127, (64,)), (400, 7, 7, (1152,)), (8, 32, 32, (16, 16)), (1, 512, 512, (150, 150)), (2, 130, 26, (128, 128)),
         (400, 8, 1, (4096,)), (1, 8, 2, (64, 64)), (1, 1030, 1, (3, 5))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("far", [1, 2, 18, 64])
@pytest.mark.parametrize("size", FIRST)
def test_first_positions_far_from_the_rest(size, far, dtype):
    """A border of other values, where every thread's sums begin."""
    n, c, groups, pos = size
    x = channels_last(n, c, (math.prod(pos),), dtype, 6, spread=False)
    x = x.clone(memory_format=torch.preserve_format)
    x[:, :, :far] += 1000.0
    mean, rstd = statistics(x, groups)
    m64, r64, sigma = statistics64(x, groups)
    # a thread's squares add up to at most 9 times its sum of squared deviations (the centre is the
    # mean of eight of its values, or of an eighth); 64 of them in fp32 come within 4 U as a rule, all
    # columns taken 6 U: 54 U, halved by the root; joins and the root itself a few U
    assert ((rstd.double() - r64).abs() <= r64 * 36 * U).all(), ((rstd / r64 - 1).abs().max() / U).item()
    assert ((mean.double() - m64).abs() <= 16 * U * (sigma + m64.abs())).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("c", [65_537, 300_001, 1_048_577, 262_144])
def test_one_group_of_very_many_channels(c, rows, dtype):
    x = channels_last(1, c, (rows,), dtype, 7, spread=False).clone(memory_format=torch.preserve_format)
    x[:, :128] += 1000.0  # where a thread's sums begin
    mean, rstd = statistics(x, 1)
    m64, r64, sigma = statistics64(x, 1)
    assert ((rstd.double() - r64).abs() <= r64 * 36 * U).all(), ((rstd / r64 - 1).abs().max() / U).item()
    assert ((mean.double() - m64).abs() <= 16 * U * (sigma + m64.abs())).all()


@pytest.mark.parametrize("size", [(1, 64, 8, (400, 400)), (1, 128, 32, (512, 512)), (2, 130, 26, (128, 128)), (4, 32, 8, (40, 40)), (25, 300, 5, (68, 3))])
@pytest.mark.parametrize("mean", [0.0, 1e3, -3e4, 1e5])
def test_deviations_of_data_far_from_zero(size, mean):
    """The mean's rounding is 1/170 of a deviation at 1e5: the squares must not feel it."""
    n, c, groups, pos = size
    x = channels_last(n, c, pos, torch.float32, 8, spread=False) + mean
    got, rstd = statistics(x, groups)
    m64, r64, sigma = statistics64(x, groups)
    # squares near the centre 4 U, joins and the root a few U, as above; the centre itself is off by U |mean| at
    # most, which squares of differences taken about it and corrected by their sum do not feel
    assert ((rstd.double() - r64).abs() <= r64 * 16 * U).all(), ((rstd / r64 - 1).abs().max() / U).item()
    assert ((got.double() - m64).abs() <= U * (m64.abs() + 2 * sigma)).all()
