"""Argument checks of the gradient-list and group-norm calls, through the C ABI and without a GPU:
a call with valid arguments gets as far as asking for the device, an invalid one does not."""
import ctypes as C
import math

import pytest
import torch

from paper_2306_06098_b200 import binding as B

FAKE = 0x7F0000000000  # never read: there is no device

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")


def tensor(numel=100, data=FAKE, dtype=0, size=(), stride=()):
    t = B.TensorDesc(data=data, numel=numel, dtype=dtype, rank=len(size))
    for k, (s, st) in enumerate(zip(size, stride)):
        t.size[k], t.stride[k] = s, st
    return t


def listed(*ts):
    return (B.TensorDesc * max(1, len(ts)))(*ts)


def norm(*ts, scale=1.0, out=FAKE, ws=FAKE, n=None):
    return B._lib.efcp_grads_norm(listed(*ts), len(ts) if n is None else n, scale, out, ws, None)


def clip(*ts, max_norm=1.0, scale=1.0, out=FAKE, ws=FAKE):
    return B._lib.efcp_grads_clip(listed(*ts), len(ts), max_norm, scale, out, ws, None)


def gather(*ts, flat=FAKE, d=100, max_norm=0.0, scale=1.0, out=None, ws=None):
    return B._lib.efcp_grads_gather(listed(*ts), len(ts), flat, d, max_norm, scale, out, ws, None)


def test_struct_sizes_match_the_header():
    assert C.sizeof(B.TensorDesc) == 8 + 8 + 4 + 4 + 8 * 8 * 2
    assert C.sizeof(B.GroupNormDesc) == 3 * 8 + 4 * 4 + 6 * 8 + 8
    assert B._lib.efcp_grads_workspace_bytes() > 0


VALID = [
    tensor(), tensor(0, None), tensor(0, None, size=(0, 3), stride=(3, 1)), tensor(7, FAKE + 2, dtype=1),
    tensor(100, size=(10, 10), stride=(1, 10)), tensor(100, size=(10, 10), stride=(20, 1)),
    tensor(1, size=(1, 1), stride=(5, 9)), tensor(1 << 40),
    tensor(32, size=(2, 2, 2, 2, 2), stride=(16, 8, 4, 2, 1)),          # merges into one dimension
    tensor(16, size=(2, 2, 2, 2), stride=(100, 30, 9, 2)),              # four that do not merge
    tensor(100, size=(10, 10), stride=(1 << 40, 1)),                    # offsets beyond 32 bits
]
INVALID = [
    tensor(-1), tensor(100, FAKE + 2), tensor(100, FAKE + 1, dtype=2), tensor(dtype=3), tensor(dtype=-1),
    tensor((1 << 40) + 1), tensor(100, size=(10, 11), stride=(11, 1)), tensor(100, size=(10, 9), stride=(9, 1)),
    tensor(100, size=(10, 10), stride=(10, -1)), tensor(100, size=(-10, -10), stride=(10, 1)),
    tensor(4, size=(1 << 62, 4), stride=(1, 1)),
    tensor(32, size=(2,) * 5, stride=(100, 40, 15, 5, 2)),              # five that do not merge
]


@pytest.mark.parametrize("i", range(len(VALID)))
def test_valid_descriptors_reach_the_device(i):
    t = VALID[i]
    assert norm(t) == B.ECUDA
    assert clip(t) == B.ECUDA
    assert gather(t, d=t.numel) == B.ECUDA


@pytest.mark.parametrize("i", range(len(INVALID)))
def test_invalid_descriptors_are_refused(i):
    t = INVALID[i]
    assert norm(t) == B.EINVAL
    assert clip(t) == B.EINVAL
    assert gather(t, d=t.numel) == B.EINVAL
    assert norm(tensor(), t) == B.EINVAL


def test_shared_elements_may_be_read_but_not_clipped():
    for t in (tensor(100, size=(10, 10), stride=(0, 1)), tensor(100, size=(10, 10), stride=(5, 1)),
              tensor(8, size=(2, 4), stride=(1, 1)), tensor(5, size=(5,), stride=(0,))):
        assert norm(t) == B.ECUDA
        assert gather(t, d=t.numel) == B.ECUDA
        assert clip(t) == B.EINVAL


def test_an_absent_gradient_needs_no_layout():
    assert gather(tensor(60), tensor(40, None)) == B.ECUDA
    assert gather(tensor(60), tensor(41, None)) == B.EINVAL  # the sum is not d
    assert norm(tensor(60), tensor(40, None)) == B.ECUDA


def test_scalars_and_pointers_of_the_list_calls():
    t = tensor()
    for s in (0.0, -1.0, math.inf, math.nan):
        assert norm(t, scale=s) == clip(t, scale=s) == gather(t, scale=s) == B.EINVAL
    for m in (0.0, -1.0, math.nan):
        assert clip(t, max_norm=m) == B.EINVAL
    assert clip(t, max_norm=math.inf) == B.ECUDA
    assert gather(t, max_norm=-1.0) == gather(t, max_norm=math.nan) == B.EINVAL
    assert norm(t, out=None) == norm(t, ws=None) == norm(t, ws=FAKE + 4) == B.EINVAL
    assert clip(t, ws=None) == B.EINVAL and clip(t, out=None) == B.ECUDA
    assert gather(t, flat=None) == gather(t, flat=FAKE + 2) == B.EINVAL
    assert gather(t, max_norm=1.0) == gather(t, out=FAKE) == B.EINVAL  # these need a workspace
    assert gather(t, max_norm=1.0, out=FAKE, ws=FAKE) == B.ECUDA
    assert norm(t, n=-1) == B.EINVAL
    assert B._lib.efcp_grads_norm(None, 1, 1.0, FAKE, FAKE, None) == B.EINVAL


def desc(**more):
    d = dict(n=2, rows=30, channels=24, groups=6, dtype=0, param_dtype=0, act=0, x_batch=720,
             x_row=24, y_batch=720, y_row=24, dy_batch=720, dy_row=24, eps=1e-5)
    d.update(more)
    return B.GroupNormDesc(**d)


def forward(d, x=FAKE, w=FAKE, b=FAKE, y=FAKE, mean=FAKE, rstd=FAKE, ws=FAKE, size=1 << 30):
    return B._lib.efcp_group_norm_forward(C.byref(d), x, w, b, y, mean, rstd, ws, size, None)


def backward(d, dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, w=FAKE, b=FAKE, dx=FAKE, dw=FAKE, db=FAKE,
             ws=FAKE, size=1 << 30):
    return B._lib.efcp_group_norm_backward(C.byref(d), dy, x, mean, rstd, w, b, dx, dw, db, ws, size, None)


def test_group_norm_descriptors():
    for ok in (desc(), desc(rows=1), desc(groups=1), desc(groups=24), desc(x_row=25, x_batch=1000),
               desc(x_batch=0), desc(dtype=1, param_dtype=2), desc(act=2), desc(eps=0.0), desc(n=1, y_batch=0),
               desc(y_row=48, y_batch=24), desc(channels=1 << 20, x_row=1 << 20, y_row=1 << 20, dy_row=1 << 20,
                                                groups=1, y_batch=30 << 20)):
        assert forward(ok) == B.ECUDA
        assert backward(ok) == B.ECUDA
        assert B._lib.efcp_group_norm_workspace_bytes(C.byref(ok), 0) > 0
        assert B._lib.efcp_group_norm_workspace_bytes(C.byref(ok), 1) > 0
    for bad in (desc(n=-1), desc(rows=0), desc(channels=0), desc(groups=0), desc(groups=5), desc(groups=-6),
                desc(dtype=3), desc(param_dtype=-1), desc(act=3), desc(eps=-1e-9), desc(eps=math.nan),
                desc(eps=math.inf), desc(rows=1 << 41), desc(n=1 << 41), desc(channels=1 << 30)):
        assert forward(bad) == B.EINVAL
        assert backward(bad) == B.EINVAL
        assert B._lib.efcp_group_norm_workspace_bytes(C.byref(bad), 0) == -1
    for bad in (desc(x_row=23), desc(y_row=23), desc(x_batch=-1), desc(y_batch=700), desc(y_batch=0),
                desc(x_row=1 << 60), desc(x_batch=1 << 60), desc(y_row=47, y_batch=24)):
        assert forward(bad) == B.EINVAL
        assert backward(bad) == B.EINVAL
    assert forward(desc(dy_row=3)) == B.ECUDA  # not looked at
    assert backward(desc(dy_row=3)) == B.EINVAL
    assert B._lib.efcp_group_norm_workspace_bytes(None, 0) == -1
    assert B._lib.efcp_group_norm_forward(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1, None) == B.EINVAL


def test_group_norm_pointers():
    d = desc()
    for k in ("x", "y", "mean", "rstd", "ws"):
        assert forward(d, **{k: None}) == B.EINVAL
        assert forward(d, **{k: FAKE + 2}) == B.EINVAL
    assert forward(d, w=None) == forward(d, b=None) == forward(d, w=None, b=None) == B.ECUDA
    assert forward(d, w=FAKE + 2) == B.EINVAL
    for k in ("x", "dy", "dx", "mean", "rstd", "ws"):
        assert backward(d, **{k: None}) == B.EINVAL
        assert backward(d, **{k: FAKE + 2}) == B.EINVAL
    for k in ("w", "b", "dw", "db"):
        assert backward(d, **{k: None}) == B.ECUDA
        assert backward(d, **{k: FAKE + 2}) == B.EINVAL
    assert forward(desc(dtype=1), x=FAKE + 2) == B.ECUDA
    assert forward(desc(n=0)) == B.OK  # nothing to do
    assert forward(desc(n=0), x=None, y=None, mean=None, rstd=None, ws=None) == B.OK


def test_layouts_of_torch_tensors():
    from paper_2306_06098_b200._marshal import as_channels_last, like_channels_last, rows_layout
    x = torch.zeros(2, 6, 5, 4)
    assert rows_layout(x) is None
    cl = x.contiguous(memory_format=torch.channels_last)
    assert rows_layout(cl) == (120, 6)
    assert rows_layout(cl[:, 1:4]) == (120, 6)
    assert rows_layout(cl[:, :, 1:3]) == (120, 6)
    assert rows_layout(cl[:, :, :, 1:3]) is None
    assert rows_layout(cl[:, :, :, :1]) == (120, 24)
    assert rows_layout(cl[1:]) == (120, 6)
    assert rows_layout(x[:, :, :1, :1]) is None
    assert rows_layout(torch.zeros(3, 7)) == (7, 7)
    assert rows_layout(torch.zeros(3, 1, 4, 4)) == (16, 1)
    assert rows_layout(torch.zeros(1, 6).expand(3, 6)) == (0, 6)
    assert rows_layout(torch.zeros(1, 6, 1).expand(2, 6, 9)) is None
    assert rows_layout(torch.zeros(0, 6, 5, 4)) == (6, 6)
    g = torch.Generator().manual_seed(0)
    for t in (torch.randn(x.shape, generator=g), cl, torch.randn(2, 6, 5, 4, generator=g)[:, :, :, 1:3],
              torch.randn(2, 6, 5, 4, 3, generator=g), torch.randn(1, 6, 1, generator=g).expand(2, 6, 9),
              torch.randn(1, generator=g).expand(2, 6, 3, 3)):
        c = as_channels_last(t)
        assert c.shape == t.shape and rows_layout(c) is not None and torch.equal(c, t)
    assert as_channels_last(cl).data_ptr() == cl.data_ptr()
    y = like_channels_last(x)
    assert y.shape == x.shape and y.is_contiguous(memory_format=torch.channels_last)
    with pytest.raises(TypeError):
        rows_layout(3)


def test_marshalling_refuses_what_it_cannot_describe():
    for bad, err in (([torch.zeros(3)], ValueError), (3, TypeError), ("abc", TypeError),
                     ([torch.zeros(3).to_sparse()], ValueError)):
        with pytest.raises(err):
            B.grad_norm(bad)
    with pytest.raises(ValueError):
        B.gather_grads([torch.zeros(3)], torch.zeros(3))
    with pytest.raises(TypeError):
        B.gather_grads([torch.zeros(3)], None)
    for call in (lambda: B.group_norm_forward(torch.zeros(2, 4, 3), 2),
                 lambda: B.group_norm_forward(torch.zeros(4), 2),
                 lambda: B.group_norm_forward(torch.zeros(2, 4, dtype=torch.float64), 2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        B.group_norm_forward(None, 2)
