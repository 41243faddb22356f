"""Argument checks of the RMS-norm and dropout calls, without a GPU: through the C ABI a call with valid arguments gets
as far as asking for the device, an invalid one does not; in Python the wrong tensors are refused."""
import ctypes as C
import math

import pytest
import torch

from paper_2306_06098_b200 import binding as B

FAKE = 0x7F0000000000  # never read: there is no device
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")
EMPTY = 1 << 40


def desc(rows=5, d=64, dtype=0, param=0, p=0.0, eps=1e-6, rng=None):
    return C.byref(B.RmsNormDesc(rows=rows, d=d, dtype=dtype, param_dtype=param, p=p, eps=eps, rng=rng))


def forward(de, x=FAKE, x_row=64, r=None, r_row=64, w=None, y=FAKE, h=None, rstd=FAKE):
    return B._lib.efcp_rms_norm_forward(de, x, x_row, r, r_row, w, y, h, rstd, None)


def quantize(de, fmt=0, block=0, x=FAKE, x_row=64, r=None, w=None, q=FAKE, s=FAKE, h=None):
    return B._lib.efcp_rms_norm_quantize(de, fmt, block, x, x_row, r, 64, w, q, s, h, None, None)


def backward(de, dy=FAKE, dy_row=64, h=FAKE, h_row=64, dh=None, dh_row=0, rstd=FAKE, w=FAKE, dx=FAKE, dr=FAKE, dw=FAKE,
             ws=FAKE, size=EMPTY):
    return B._lib.efcp_rms_norm_backward(de, dy, dy_row, h, h_row, dh, dh_row, rstd, w, dx, dr, dw, ws, size, None)


def drop(de, x=FAKE, x_row=64, r=None, r_row=64, y=FAKE):
    return B._lib.efcp_dropout(de, x, x_row, r, r_row, y, None)


CALLS = (forward, quantize, backward, drop)


@no_gpu
def test_valid_calls_reach_the_device():
    assert C.sizeof(B.RmsNormDesc) == 2 * 8 + 2 * 4 + 8 + 2 * 8 + 8 + 8
    for call in CALLS:
        for de in (desc(), desc(p=0.0, dtype=1, param=2), desc(d=1), desc(d=(1 << 30) - 1, rows=1), desc(eps=0.0),
                   desc(rows=1 << 34)):
            assert call(de) == B.ECUDA
        assert call(desc(rows=0)) == B.OK or call is backward
    for call in (forward, drop):
        assert call(desc(p=0.5, rng=FAKE), **({"h": FAKE} if call is forward else {})) == B.ECUDA
        assert call(desc(), x_row=0) == B.ECUDA  # one row again and again
    assert forward(desc(), r=FAKE, h=FAKE, rstd=None) == B.ECUDA
    assert backward(desc(), dw=None, ws=None, size=0) == B.ECUDA
    assert backward(desc(), dx=None, dr=None) == B.ECUDA
    assert backward(desc(), dx=None, dr=None, dw=None) == B.OK
    for fmt in (0, 1):
        for block in (0, 32, 64, 128):
            assert quantize(desc(), fmt, block) == B.ECUDA


@no_gpu
def test_invalid_calls_are_refused():
    for call in CALLS:
        for de in (desc(rows=-1), desc(d=0), desc(d=1 << 30), desc(rows=(1 << 35), d=64), desc(dtype=3), desc(param=-1),
                   desc(p=-0.1), desc(p=1.1), desc(p=math.nan), desc(eps=-1.0), desc(eps=math.inf), desc(eps=math.nan),
                   desc(p=0.5, rng=FAKE + 4), None):
            assert call(de) == B.EINVAL
    for more in (dict(x=None), dict(x=FAKE + 2), dict(x_row=-1), dict(x_row=1 << 50), dict(r=FAKE), dict(r=FAKE + 1, h=FAKE),
                 dict(w=FAKE + 2), dict(y=None), dict(y=FAKE + 1), dict(rstd=FAKE + 2)):
        assert forward(desc(), **more) == B.EINVAL
    assert forward(desc(p=0.5)) == B.EINVAL  # h is missing
    for more in (dict(fmt=2), dict(fmt=-1), dict(block=16), dict(block=-32), dict(q=None), dict(s=None), dict(s=FAKE + 2)):
        assert quantize(desc(), **more) == B.EINVAL
    for more in (dict(dy=None), dict(dy=FAKE + 1), dict(h=None), dict(h_row=-1), dict(dh=FAKE + 2), dict(dh=FAKE, dh_row=-1),
                 dict(rstd=None), dict(w=FAKE + 1), dict(dx=FAKE + 1), dict(dr=FAKE + 3), dict(dw=FAKE + 2), dict(ws=None),
                 dict(ws=FAKE + 8)):
        assert backward(desc(), **more) == B.EINVAL
    for more in (dict(x=None), dict(x=FAKE + 1), dict(x_row=-3), dict(r=FAKE + 2), dict(r=FAKE, r_row=-1), dict(y=None)):
        assert drop(desc(), **more) == B.EINVAL


def test_the_workspace_grows_with_the_row():
    size = lambda *a: B._lib.efcp_rms_norm_workspace_bytes(desc(*a))  # noqa: E731
    assert size(1, 8) >= 32 and size(1000, 4096) >= 148 * 4096 * 4 and size(2, 40000) >= 40000 * 4
    assert size(-1, 8) == -1 and size(1, 0) == -1


@no_gpu
def test_tensors_that_are_refused():
    x = torch.ones(4, 8)
    one = torch.ones(4)
    rng = (1, 2)
    for bad in (lambda: B.rms_norm_forward(x), lambda: B.dropout(x, 0.5, rng), lambda: B.rms_norm_quantize(x),
                lambda: B.rms_norm_backward(x, x, one)):
        with pytest.raises(ValueError, match="CUDA"):
            bad()
    for bad in (torch.ones(4, 8, dtype=torch.float64), torch.tensor(1.0), torch.ones(4, 8).to_sparse()):
        for call in (lambda: B.rms_norm_forward(bad), lambda: B.dropout(bad, 0.5, rng)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: B.rms_norm_forward(3), lambda: B.dropout(None, 0.5, rng), lambda: B.rms_norm_backward(x, x, None)):
        with pytest.raises(TypeError):
            call()


class OtherStream:
    """What a stream of another device looks like; entering it would need that device."""
    device = torch.device("cuda", 7)


@pytest.mark.parametrize("k", range(4))
def test_a_stream_of_another_device_is_refused(k):
    t, s = torch.ones(6, 8), OtherStream()
    call = [lambda: B.rms_norm_forward(t, stream=s), lambda: B.rms_norm_backward(t, t, t, stream=s),
            lambda: B.rms_norm_quantize(t, stream=s), lambda: B.dropout(t, 0.5, (1, 2), stream=s)][k]
    with pytest.raises(ValueError, match="stream"):
        call()


@pytest.mark.gpu
def test_arguments_that_are_refused():
    x, w, one = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda"), torch.ones(4, device="cuda")
    half = x.half()
    refused = [
        lambda: B.rms_norm_forward(x, w.cpu()), lambda: B.rms_norm_forward(x, w[:4]), lambda: B.rms_norm_forward(x, w.double()),
        lambda: B.rms_norm_forward(x, torch.ones(16, device="cuda")[::2]), lambda: B.rms_norm_forward(x, None, 1e-6, half),
        lambda: B.rms_norm_forward(x, None, 1e-6, x[:2]), lambda: B.rms_norm_forward(x, None, 1e-6, x.cpu()),
        lambda: B.rms_norm_forward(x, p=0.5, rng=torch.zeros(2, device="cuda")),
        lambda: B.rms_norm_forward(x, p=0.5, rng=torch.zeros(2, dtype=torch.int64)),
        lambda: B.rms_norm_forward(x, p=0.5, rng=torch.zeros(3, dtype=torch.int64, device="cuda")),
        lambda: B.rms_norm_backward(half, x, one), lambda: B.rms_norm_backward(x, x, one[:2]),
        lambda: B.rms_norm_backward(x, x, one.double()), lambda: B.rms_norm_backward(x, x, one, w, half),
        lambda: B.rms_norm_quantize(x, block=16), lambda: B.rms_norm_quantize(x, format="e5m2"),
        lambda: B.rms_norm_quantize(x, residual=half), lambda: B.dropout(x, 0.5, (1, 2), half),
        lambda: B.dropout(x, 0.5, torch.zeros(2, device="cuda"))]
    for k, call in enumerate(refused):
        with pytest.raises(ValueError):
            call()
            print(k)
    for call in (lambda: B.dropout(x, 0.5, None), lambda: B.dropout(x, 0.5, (1,)), lambda: B.dropout(x, 0.5, (1.0, 2)),
                 lambda: B.rms_norm_forward(x, p=0.5)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.dropout(x, 1.5, (1, 2)), lambda: B.dropout(x, -0.5, (1, 2)), lambda: B.rms_norm_forward(x, eps=-1.0),
                 lambda: B.rms_norm_forward(torch.ones(4, 0, device="cuda")), lambda: B.rms_norm_forward(x, p=float("nan"))):
        with pytest.raises(B.EfcpError):
            call()
