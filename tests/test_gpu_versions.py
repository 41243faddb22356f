"""What autograd is told of tensors that the list calls write: one change for each that was written, none where a call was
refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def values(n, seed):
    return torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def test_a_refused_call_changes_no_version():
    from paper_2306_06098_b200 import binding as B
    g = [values(100, 1), values(50, 2)]
    versions = [t._version for t in g]
    for bad, kind in ((lambda: B.clip_grads(g + [torch.zeros(3)], 1.0), ValueError), (lambda: B.clip_grads(g + [None], 1.0), TypeError),
                      (lambda: B.clip_grads(g + [g[0].double()], 1.0), ValueError), (lambda: B.clip_grads(g, -1.0), B.EfcpError),
                      (lambda: B.clip_grads(g + [values(1, 3).expand(5)], 1.0), B.EfcpError),
                      (lambda: B.clip_grads(g, 1.0, out=torch.zeros(2, device="cuda")), ValueError)):
        with pytest.raises(kind):
            bad()
        assert [t._version for t in g] == versions
    flat, out = torch.empty(150, device="cuda"), torch.zeros((), device="cuda")
    versions = flat._version, out._version
    with pytest.raises(B.EfcpError):
        B.gather_grads(g + [3], flat, out=out)
    assert (flat._version, out._version) == versions


def test_every_output_counts_as_changed():
    from paper_2306_06098_b200 import binding as B
    g = [values(100, 1), values(50, 2)]
    flat, out = torch.empty(150, device="cuda"), torch.zeros((), device="cuda")
    B.grad_norm(g, out=out)
    assert out._version == 1 and [t._version for t in g] == [0, 0]
    B.gather_grads(g, flat, out=out)
    assert (out._version, flat._version) == (2, 1)
    B.gather_grads(g, flat)
    assert (out._version, flat._version) == (2, 2)
    B.clip_grads(g, 1.0, out=out)
    assert out._version == 3 and [t._version for t in g] == [1, 1]


def test_a_result_that_backward_needs_may_not_be_overwritten():
    from paper_2306_06098_b200 import binding as B
    flat = torch.ones(150, device="cuda")
    w = torch.ones(150, device="cuda", requires_grad=True)
    loss = (w * flat).sum()  # keeps flat
    B.gather_grads([values(150, 1)], flat)
    with pytest.raises(RuntimeError):
        loss.backward()


def test_tensors_of_inference_mode():
    from paper_2306_06098_b200 import binding as B
    with torch.inference_mode():
        g = values(100, 1).clone()
        out = torch.zeros((), device="cuda")
        before = g.clone()
        n = B.clip_grads([g], 1.0, out=out).item()
        assert n > 1 and not torch.equal(g, before)
    kept = g.clone()
    with pytest.raises(RuntimeError):  # as torch's own operations in place
        B.clip_grads([g], 0.5)
    torch.cuda.synchronize()
    assert torch.equal(g, kept)
    assert abs(B.grad_norm([g], out=out).item() - 1.0) < 1e-5  # reading them and writing the norm stays open
