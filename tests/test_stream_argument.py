"""`stream=` of the list and group-norm calls: a stream of another device than the tensors' would not be the one the
work runs on."""
import pytest
import torch

from paper_2306_06098_b200 import binding as B


class OtherStream:
    """What a stream of another device looks like; entering it would need that device."""
    device = torch.device("cuda", 7)


def calls(t, stream):
    x = t.view(1, -1, 1)
    one = torch.ones(1)
    return [lambda: B.grad_norm([t], stream=stream), lambda: B.grad_norm([t], out=one, stream=stream),
            lambda: B.clip_grads((t,), 1.0, stream=stream), lambda: B.gather_grads([t], t.clone(), stream=stream),
            lambda: B.gather_grads([6], t.clone(), stream=stream), lambda: B.group_norm_forward(x, 2, stream=stream),
            lambda: B.group_norm_backward(x, x, one, one, 2, stream=stream)]


@pytest.mark.parametrize("k", range(7))
def test_a_stream_of_another_device_is_refused(k):
    with pytest.raises(ValueError, match="stream"):
        calls(torch.ones(6), OtherStream())[k]()


@pytest.mark.gpu
def test_a_stream_of_the_tensors_device():
    t = torch.ones(6, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    n = B.grad_norm([t], stream=side)
    side.synchronize()
    assert abs(n.item() - 6 ** 0.5) < 1e-6
