"""Key rows that do not count (k_used) have no gradient: the binding's own dk and dv are zero there, whatever its memory held before."""
import pytest
import torch

import paper_2506_21411_amd as dchag

from .test_gpu_attend import LOG, Problem, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("used", [[150, 1], [0, 70], [200, 130]], ids=str)
def test_gradient_of_keys_that_do_not_count(dtype, used):
    p = Problem(dtype, 2, 1, 64, [90, 60], [200, 130], causal=True, borders=LOG, used=used, seed=52, tail=0)
    q, k, v, dout, kw = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda(), p.kw()
    out, lse = dchag.dchag_attend(q, k, v, dev(p.qs), dev(p.ks), **kw)
    left = [torch.full_like(t, float("nan")) for t in (q, k, v, k, v)]
    del left                                                       # memory for the call's own tensors to be made of
    _, dk, dv, _ = dchag.dchag_attend_backward(q, k, v, out, lse, dout, dev(p.qs), dev(p.ks), **kw)
    rows = (~p.in_k).cuda()
    assert bool((dk[rows] == 0).all()) and bool((dv[rows] == 0).all())
    want = p.want()
    for name, got in (("dk", dk), ("dv", dv)):
        value, bound = (x[p.in_k] for x in want[name])
        p_in = got[p.in_k.cuda()].double().cpu()
        assert bool(((p_in - value).abs() <= bound + 1e-30).all()), name
