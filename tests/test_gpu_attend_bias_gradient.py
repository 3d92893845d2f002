"""The bias gradient within bounds that zeros, or sums without the far pairs, do not pass (test_spatial_bias_reference.py sees to that)."""
import pytest

from . import spatial_bias_reference as sums
from . import spatial_reference as ref
from .bias_gradient_cases import CASES
from .test_gpu_attend import Problem, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(CASES))
def test_bias_gradient(name):
    say(f"bias gradient {name} {CASES[name]}")
    p = Problem(tail=0, **CASES[name])
    value, bound, _ = sums.bias_gradient(p.q, p.k, p.v, p.qs, p.ks, p.bias, p.borders, p.dout, p.causal, p.used)
    got = p.run()["dbias"]
    off = ((got.double().cpu() - value).abs() / bound.clamp(min=1e-30)).max()
    say(f"largest error {float(off):.2f} of its bound")
    ref.check("dbias", got, value, bound)
