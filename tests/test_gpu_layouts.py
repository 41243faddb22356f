"""Layouts that a caller of the C ABI may use and torch does not make by itself, and parameters kept channels last."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("n,rows,c,groups", [(2, 30, 24, 6), (5, 400, 16, 4), (3, 17_000, 64, 32), (4, 9, 33, 11)])
def test_samples_inside_rows(n, rows, c, groups, act):
    """Outputs and inputs laid out (rows, samples, channels)."""
    from paper_2306_06098_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(n, rows, c, generator=g, device="cuda") for _ in range(2))
    w, b = 1 + 0.3 * torch.randn(c, generator=g, device="cuda"), 0.3 * torch.randn(c, generator=g, device="cuda")
    name = B.ACTS[act]
    want = B.group_norm_forward(x.permute(0, 2, 1), groups, w, b, 1e-5, name)
    wantg = B.group_norm_backward(dy.permute(0, 2, 1), x.permute(0, 2, 1), want[1], want[2], groups, w, b, name)
    xi, di = (t.transpose(0, 1).contiguous() for t in (x, dy))
    y, dx = (torch.full((rows * n * c + 8,), -7.0, device="cuda") for _ in range(2))
    d = B.GroupNormDesc(n=n, rows=rows, channels=c, groups=groups, dtype=B.F32, param_dtype=B.F32, act=act, x_batch=c, x_row=n * c,
                        y_batch=c, y_row=n * c, dy_batch=c, dy_row=n * c, eps=1e-5)
    mean, rstd = (torch.empty(n, groups, device="cuda") for _ in range(2))
    dw, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    for back in (0, 1):
        size = B._lib.efcp_group_norm_workspace_bytes(C.byref(d), back)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        if back:
            rc = B._lib.efcp_group_norm_backward(C.byref(d), di.data_ptr(), xi.data_ptr(), mean.data_ptr(), rstd.data_ptr(), w.data_ptr(),
                                                 b.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.data_ptr(), size, st)
        else:
            rc = B._lib.efcp_group_norm_forward(C.byref(d), xi.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), mean.data_ptr(),
                                                rstd.data_ptr(), ws.data_ptr(), size, st)
        assert rc == B.OK
    for got, ref in ((y, want[0]), (dx, wantg[0])):
        assert torch.equal(got[:rows * n * c].view(rows, n, c).permute(1, 2, 0), ref)
        assert (got[rows * n * c:] == -7).all()
    for got, ref in ((mean, want[1]), (rstd, want[2]), (dw, wantg[1]), (db, wantg[2])):
        assert torch.equal(got, ref)


def test_parameters_that_were_channels_last():
    """The optimizer lays them out in the order of their indices; values, gradients and steps stay the same."""
    from paper_2306_06098_b200.optim import SparseMFAC

    def model(fmt):
        torch.manual_seed(0)
        return torch.nn.Sequential(torch.nn.Conv2d(4, 16, 3), torch.nn.ReLU(), torch.nn.Conv2d(16, 8, 3)).to(
            device="cuda", memory_format=fmt)

    a, b = model(torch.channels_last), model(torch.contiguous_format)
    assert not a[0].weight.is_contiguous()
    opt_a, opt_b = (SparseMFAC(m.parameters(), lr=0.1, m=4, density=0.1, damp=1e-3, max_grad_norm=0.5) for m in (a, b))
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        for p, q in zip(a.parameters(), b.parameters()):
            assert torch.equal(p, q)
            v = torch.randn(p.shape, generator=g, device="cuda")
            p.grad = v.contiguous(memory_format=torch.channels_last) if v.dim() == 4 else v
            q.grad = v.clone()
        opt_a.step()
        opt_b.step()
        assert torch.equal(opt_a._g, opt_b._g) and torch.equal(opt_a._theta, opt_b._theta)
    # and through autograd
    x = torch.randn(2, 4, 9, 9, generator=g, device="cuda").contiguous(memory_format=torch.channels_last)
    opt_a.zero_grad()
    a(x).square().sum().backward()
    flat = torch.cat([p.grad.reshape(-1) for p in a.parameters()])
    opt_a.max_grad_norm = 0.0
    opt_a.step()
    assert torch.equal(opt_a._g, flat)
