"""Tensors of more than 2^31 elements, whose offsets leave 32 bits: lists of gradients and group norm."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LONG = 1 << 31


@pytest.fixture(autouse=True)
def room():
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    yield
    torch.cuda.empty_cache()


def fill(t, seed):
    return t.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


def sumsq64(flat):
    return sum(flat[k:k + (1 << 27)].double().square().sum().item() for k in range(0, flat.numel(), 1 << 27))


def same(a, b):
    return all(torch.equal(a[k:k + (1 << 28)], b[k:k + (1 << 28)]) for k in range(0, a.numel(), 1 << 28))


def test_one_after_another():
    from paper_2306_06098_b200 import binding as B
    n = LONG + 12_345
    ts = [fill(torch.empty(n, dtype=torch.float16, device="cuda"), 1), fill(torch.empty(77, device="cuda"), 2)]
    n64 = math.sqrt(sum(sumsq64(t) for t in ts))
    assert abs(B.grad_norm(ts).item() - n64) <= 6 * U * n64
    flat = torch.empty(n + 77, device="cuda")
    B.gather_grads(ts, flat)
    assert torch.equal(flat[n:], ts[1])
    assert all(torch.equal(flat[k:k + (1 << 28)], ts[0][k:k + (1 << 28)].float()[:n - k]) if k + (1 << 28) <= n else
               torch.equal(flat[k:n], ts[0][k:].float()) for k in range(0, n, 1 << 28))
    kept = ts[0][LONG - 5:].clone()
    B.clip_grads(ts, 0.5 * n64)
    want = kept.double() * 0.5
    assert ((ts[0][LONG - 5:].double() - want).abs() <= want.abs() * (2.0 ** -11 + 8 * U) + 2.0 ** -25).all()


def test_transposed():
    """Positions from divisions of 64 bits."""
    from paper_2306_06098_b200 import binding as B
    a, b = 46_349, 46_337
    base = fill(torch.empty(a, b, dtype=torch.bfloat16, device="cuda"), 3)
    t = base.t()
    assert t.numel() > LONG
    n64 = math.sqrt(sumsq64(base.view(-1)))
    assert abs(B.grad_norm([t]).item() - n64) <= 6 * U * n64
    wide = torch.empty(a, b + 3, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:] = base
    for s in (t, wide[:, 3:].t()):  # the second has gaps: every position comes from divisions in the norm too
        assert abs(B.grad_norm([s]).item() - n64) <= 6 * U * n64
        flat = torch.empty(t.numel(), device="cuda")
        B.gather_grads([s], flat)
        for k in range(0, b, 4096):
            assert torch.equal(flat.view(b, a)[k:k + 4096], t[k:k + 4096].float())
        del flat
    kept = base[-3:].clone()
    B.clip_grads([wide[:, 3:].t()], 0.25 * n64)
    want = kept.double() * 0.25
    assert ((wide[-3:, 3:].double() - want).abs() <= want.abs() * (2.0 ** -8 + 8 * U)).all()


# many small samples (each on chip), few large ones, one whose rows alone are more than 2^31 elements
@pytest.mark.parametrize("n,pos", [(10_703, (56, 56)), (17, (1408, 1408)), (1, (5801, 5801))])
def test_group_norm(n, pos):
    from paper_2306_06098_b200 import binding as B
    c, groups = 64, 32
    x = fill(torch.empty(n, *pos, c, dtype=torch.bfloat16, device="cuda"), 4).permute(0, 3, 1, 2)
    assert x.numel() > LONG
    dy = fill(torch.empty(n, *pos, c, dtype=torch.bfloat16, device="cuda"), 5).permute(0, 3, 1, 2)
    g = torch.Generator(device="cuda").manual_seed(6)
    w, b = 1 + 0.3 * torch.randn(c, generator=g, device="cuda"), 0.3 * torch.randn(c, generator=g, device="cuda")
    y, mean, rstd = B.group_norm_forward(x, groups, w, b, 1e-5, "none")
    dx, dw, db = B.group_norm_backward(dy, x, mean, rstd, groups, w, b, "none")
    rows, per = pos[0] * pos[1], c // groups
    dw64, db64 = torch.zeros(c, dtype=torch.float64, device="cuda"), torch.zeros(c, dtype=torch.float64, device="cuda")
    step = 1 << 20
    for k in range(n):
        whole = k in (0, 1, n - 2, n - 1) or n <= 17
        if not whole:
            continue
        v, d = x[k].permute(1, 2, 0).reshape(rows, c), dy[k].permute(1, 2, 0).reshape(rows, c)
        parts = range(0, rows, step)
        m64 = sum(v[i:i + step].double().view(-1, groups, per).sum((0, 2)) for i in parts) / (rows * per)
        m2 = sum((v[i:i + step].double().view(-1, groups, per) - m64[:, None]).square().sum((0, 2)) for i in parts)
        r64 = (m2 / (rows * per) + 1e-5).rsqrt()
        assert ((mean[k].double() - m64).abs() <= 8 * U).all()
        assert ((rstd[k].double() - r64).abs() <= 16 * U * r64).all()
        a64 = b64 = 0
        for i in parts:
            h = ((v[i:i + step].double().view(-1, groups, per) - m64[:, None]) * r64[:, None]).view(-1, c)
            e = d[i:i + step].double()
            a64 = a64 + (e * w).view(-1, groups, per).sum((0, 2))
            b64 = b64 + (e * w * h).view(-1, groups, per).sum((0, 2))
            if n <= 17:
                dw64 += (e * h).sum(0)
                db64 += e.sum(0)
        for i in (0, (rows - 1) // 2, max(0, rows - 3000)):  # rows at both ends and in between
            s = slice(i, min(rows, i + 3000))
            h = ((v[s].double().view(-1, groups, per) - m64[:, None]) * r64[:, None]).view(-1, c)
            z = h * w + b
            got = y[k].permute(1, 2, 0).reshape(rows, c)[s].double()
            assert ((got - z).abs() <= 2.0 ** -8 * z.abs() + 64 * U * (1 + h.abs())).all()
            e = d[s].double() * w
            q = (e.view(-1, groups, per) - a64[:, None] / (rows * per)
                 - h.view(-1, groups, per) * (b64 / (rows * per))[:, None]) * r64[:, None]
            got = dx[k].permute(1, 2, 0).reshape(rows, c)[s].double().view(-1, groups, per)
            mag = r64[:, None] * (e.abs().view(-1, groups, per) + 1 + h.abs().view(-1, groups, per))
            assert ((got - q).abs() <= 2.0 ** -8 * q.abs() + 64 * U * mag).all()
    if n <= 17:
        # n rows terms of about 1, added in fp32 over short runs, then in 64 bits
        lim = 64 * U * math.sqrt(n * rows) + 2e-6 * math.sqrt(n * rows)
        assert ((dw.double() - dw64).abs() <= lim + 4 * U * dw64.abs()).all()
        assert ((db.double() - db64).abs() <= lim + 4 * U * db64.abs()).all()
