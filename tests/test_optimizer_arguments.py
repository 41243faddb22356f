"""Scalars of the optimizer front end are refused when it is made, not at its first step."""
import math

import pytest
import torch


@pytest.mark.parametrize("scale", [0.0, -1.0, math.inf, math.nan])
def test_grad_scale_has_to_be_finite_and_positive(scale):
    from paper_2306_06098_b200.optim import SparseMFAC
    with pytest.raises(ValueError, match="grad_scale"):
        SparseMFAC([torch.nn.Parameter(torch.zeros(3))], lr=0.1, grad_scale=scale)


@pytest.mark.parametrize("norm", [-1.0, math.nan])
def test_max_grad_norm_has_to_be_a_number_of_0_or_more(norm):
    from paper_2306_06098_b200.optim import SparseMFAC
    with pytest.raises(ValueError, match="max_grad_norm"):
        SparseMFAC([torch.nn.Parameter(torch.zeros(3))], lr=0.1, max_grad_norm=norm)
