"""Argument checks of the RMS-norm, dropout and cross-entropy calls, without a GPU: through the C ABI a call with valid arguments gets
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


# ------------------------------------------------------------------ linear cross entropy
def loss_desc(tokens=5, vocab=100, d=64, hidden_row=64, weight_row=64, ignore=-100, dtype=1, reduction=0):
    return C.byref(B.CrossEntropyDesc(tokens, vocab, d, hidden_row, weight_row, ignore, dtype, reduction))


def loss_forward(de, h=FAKE, w=FAKE, t=FAKE, out=FAKE, lse=FAKE, ws=FAKE, size=EMPTY):
    return B._lib.efcp_cross_entropy_forward(de, h, w, t, out, lse, ws, size, None)


def loss_backward(de, g=FAKE, step=1, h=FAKE, w=FAKE, t=FAKE, lse=FAKE, dh=FAKE, dw=FAKE, ws=FAKE, size=EMPTY):
    return B._lib.efcp_cross_entropy_backward(de, g, step, h, w, t, lse, dh, dw, ws, size, None)


@no_gpu
def test_cross_entropy_calls():
    assert C.sizeof(B.CrossEntropyDesc) == 6 * 8 + 2 * 4
    for call in (loss_forward, loss_backward):
        for de in (loss_desc(), loss_desc(dtype=0), loss_desc(dtype=2, reduction=1), loss_desc(d=1), loss_desc(vocab=1),
                   loss_desc(hidden_row=0), loss_desc(weight_row=63), loss_desc(ignore=2 ** 62)):
            assert call(de) == B.ECUDA
        for de in (loss_desc(tokens=-1), loss_desc(tokens=1 << 30), loss_desc(vocab=0), loss_desc(vocab=1 << 30), loss_desc(d=0),
                   loss_desc(d=1 << 24), loss_desc(hidden_row=-1), loss_desc(weight_row=-1), loss_desc(weight_row=1 << 33),
                   loss_desc(dtype=3), loss_desc(dtype=-1), loss_desc(reduction=3), loss_desc(reduction=-1),
                   loss_desc(tokens=1 << 29, d=1 << 20), None):
            assert call(de) == B.EINVAL
            if de is not None:
                assert B._lib.efcp_cross_entropy_workspace_bytes(de, FAKE, 0) == -1
        for more in (dict(h=None), dict(h=FAKE + 1), dict(w=None), dict(w=FAKE + 1), dict(t=None), dict(t=FAKE + 4),
                     dict(lse=None), dict(lse=FAKE + 2), dict(ws=None), dict(ws=FAKE + 128)):
            assert call(loss_desc(), **more) == B.EINVAL
        for tokens in (5, 500):
            need = B._lib.efcp_cross_entropy_workspace_bytes(loss_desc(tokens=tokens), FAKE, call is loss_backward)
            assert call(loss_desc(tokens=tokens), size=need - 1) == B.ENOMEM
    assert loss_forward(loss_desc(), out=None) == loss_forward(loss_desc(), out=FAKE + 2) == B.EINVAL
    assert loss_forward(loss_desc(tokens=0), h=None, t=None, out=None, lse=None) == B.OK
    assert loss_forward(loss_desc(tokens=0, reduction=1), out=None) == B.EINVAL
    for more in (dict(g=None), dict(g=FAKE + 2), dict(step=-1), dict(dh=FAKE + 1), dict(dw=FAKE + 1)):
        assert loss_backward(loss_desc(), **more) == B.EINVAL
    assert loss_backward(loss_desc(), dh=None) == loss_backward(loss_desc(), dw=None) == B.ECUDA
    assert loss_backward(loss_desc(), dh=None, dw=None) == B.OK


def test_the_cross_entropy_workspace():
    size = lambda back, w=FAKE, **k: B._lib.efcp_cross_entropy_workspace_bytes(loss_desc(**k), w, back)  # noqa: E731
    logits = 16384 * 64000 * 2
    for back in (0, 1):
        assert 0 < size(back, tokens=16384, vocab=64000) < logits / 4  # the logits are not kept
        weight = 64000 * 64 * 2
        for more in (dict(w=FAKE + 2), dict(weight_row=67)):  # a copy of the weight that can be read by tiles
            assert size(back, tokens=9, vocab=64000, **more) - size(back, tokens=9, vocab=64000) >= weight
            assert size(back, tokens=8, vocab=64000, **more) == size(back, tokens=8, vocab=64000) < weight  # read where it lies
    # two pieces of 256 columns at least, rows of both kinds
    assert size(1, tokens=1 << 20, vocab=64000) - (1 << 20) * 64 * 6 < 2 * 2 * (1 << 20) * 256 + (64 << 20)


@no_gpu
def test_cross_entropy_tensors_that_are_refused():
    h, w, t = torch.ones(4, 8), torch.ones(5, 8), torch.zeros(4, dtype=torch.int64)
    good = (h, w, t)
    with pytest.raises(ValueError, match="CUDA"):
        B.cross_entropy_forward(*good)
    for bad in ((h.double(), w.double(), t), (h, w.half(), t), (h, w[:, :7], t), (h, w[0], t), (h, w, t[:3]), (h, w, t.int()),
                (torch.tensor(1.0), w, t), (h, w, t[None])):
        with pytest.raises(ValueError):
            B.cross_entropy_forward(*bad)
    for bad in ((None, w, t), (h, 3, t), (h, w, [1, 2, 3, 4])):
        with pytest.raises(TypeError):
            B.cross_entropy_forward(*bad)
    for call in (lambda s: B.cross_entropy_forward(*good, stream=s),
                 lambda s: B.cross_entropy_backward(torch.ones(()), *good, torch.ones(4), stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(OtherStream())


@pytest.mark.gpu
def test_cross_entropy_arguments_that_are_refused():
    h, w, t = torch.ones(4, 8, device="cuda"), torch.ones(5, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    one, lse = torch.ones((), device="cuda"), torch.ones(4, device="cuda")
    for call in (lambda: B.cross_entropy_forward(h, w, t, -100, "average"), lambda: B.cross_entropy_forward(h, w.cpu(), t),
                 lambda: B.cross_entropy_forward(h, w, t.cpu()), lambda: B.cross_entropy_backward(one, h, w, t, lse[:3]),
                 lambda: B.cross_entropy_backward(one, h, w, t, lse.double()), lambda: B.cross_entropy_backward(lse, h, w, t, lse),
                 lambda: B.cross_entropy_backward(one, h, w, t, lse, -100, "none"),
                 lambda: B.cross_entropy_backward(one.double(), h, w, t, lse)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.EfcpError):
        B.cross_entropy_forward(h, w[:0], t)
    with pytest.raises(B.EfcpError):
        B.cross_entropy_forward(h[:, :0], w[:, :0], t)
