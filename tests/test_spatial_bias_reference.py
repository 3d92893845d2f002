"""The bounds of the bias gradient's tests: they follow the same 64-bit values, and a gradient that lost something does not pass them."""
import pytest
import torch

from . import spatial_bias_reference as sums
from . import spatial_reference as ref
from .bias_gradient_cases import CASES
from .test_gpu_attend import Problem


@pytest.mark.parametrize("name", list(CASES))
def test_lost_sums_do_not_pass(name):
    p = Problem(tail=0, **CASES[name])
    value, bound, near = sums.bias_gradient(p.q, p.k, p.v, p.qs, p.ks, p.bias, p.borders, p.dout, p.causal, p.used)
    some = value != 0                                              # a bucket without a pair is 0 whatever happens
    zeros = (value.abs() > bound)[some].double().mean()
    assert zeros > 0.95, f"zeros pass for {1 - zeros:.1%} of the entries"
    side = len(p.borders) + 1
    for last in [side - 1] + ([] if p.causal else [2 * side - 1]):
        lost = ((value - near).abs() > bound)[:, last][some[:, last]].double()
        assert lost.numel() == 0 or lost.mean() > 0.85, f"bucket {last}: without its far pairs it passes for {1 - lost.mean():.1%} of the heads"


@pytest.mark.parametrize("name", ["few rows", "counted keys", "more keys"])
def test_values_are_the_other_form_s(name):
    p = Problem(tail=0, **CASES[name])
    value, _, _ = sums.bias_gradient(p.q, p.k, p.v, p.qs, p.ks, p.bias, p.borders, p.dout, p.causal, p.used)
    assert torch.allclose(value, p.want()["dbias"][0], rtol=1e-9, atol=1e-9)
