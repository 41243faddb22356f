"""Gradients that the optimizer front end has always taken: lazily negated views too."""
import pytest
import torch


def negated(n, seed, device="cpu"):
    """An fp32 tensor whose sign is a flag of the view, as the imaginary part of a conjugate."""
    z = torch.randn(n, 2, generator=torch.Generator().manual_seed(seed)).to(device)
    t = torch.view_as_complex(z).conj().imag
    assert t.is_neg()
    return t


def test_a_lazily_negated_gradient_is_resolved():
    from paper_2306_06098_b200.optim import SparseMFAC
    for make in (lambda: negated(6, 1), lambda: negated(6, 1).view(2, 3).t(), lambda: negated(64, 2).view(2, 2, 2, 2, 2, 2).permute(5, 4, 3, 2, 1, 0)):
        p = torch.nn.Parameter(torch.zeros(make().shape))
        p.grad = make()
        g = SparseMFAC._gradient(p)
        assert not g.is_neg() and torch.equal(g, p.grad)


@pytest.mark.gpu
def test_a_step_with_a_lazily_negated_gradient():
    from paper_2306_06098_b200.optim import SparseMFAC
    a, b = (torch.nn.Parameter(torch.ones(50, device="cuda")) for _ in range(2))
    opt_a, opt_b = (SparseMFAC([p], lr=0.1, m=4, density=0.2, damp=1e-3) for p in (a, b))
    for t in range(5):
        a.grad = negated(50, t, "cuda")
        b.grad = a.grad.resolve_neg()
        assert a.grad.is_neg() and not b.grad.is_neg()
        opt_a.step()
        opt_b.step()
        assert torch.equal(opt_a._g, b.grad) and torch.equal(a, b)
