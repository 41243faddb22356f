"""Gradients that are zero in most rows, as an embedding's are: exact zeros, of both signs, beside values whose squares
vanish in fp32."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def rows(n, width, live, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.zeros((n, width), device="cuda")
    at = torch.randperm(n, generator=g, device="cuda")[:live]
    t[at] = size * torch.randn((live, width), generator=g, device="cuda")
    return t.to(dtype)


@pytest.mark.parametrize("size", [1.0, 1e-30, 1e-40])
@pytest.mark.parametrize("live", [0, 1, 40, 500])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_and_gather(dtype, live, size):
    from paper_2306_06098_b200 import binding as B
    ts = [rows(500, 771, live, dtype, 1, size), rows(3000, 64, min(live, 30), torch.float32, 2, size),
          -rows(64, 512, 0, dtype, 3)]  # -0.0 throughout
    n64 = math.sqrt(sum(t.double().square().sum().item() for t in ts))
    d = sum(t.numel() for t in ts)
    flat = torch.empty(d, device="cuda")
    # the norm's sums of at most 8 squares in fp32, then 64 bits; its rounding to fp32
    tol = 6 * U * n64 + 2.0 ** -149
    assert abs(B.grad_norm(ts).item() - n64) <= tol
    assert abs(B.gather_grads(ts, flat, norm=True).item() - n64) <= tol
    want = torch.cat([t.reshape(-1).float() for t in ts])
    assert torch.equal(flat.view(torch.int32), want.view(torch.int32))
    assert abs(B.clip_grads(ts, 2.0 * max(n64, 1e-30)).item() - n64) <= tol
    assert torch.equal(torch.cat([t.reshape(-1).float() for t in ts]).view(torch.int32), want.view(torch.int32))
