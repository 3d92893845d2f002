"""dq, dk and dv do not depend on whether the bias gradient is wanted."""
import pytest
import torch

import paper_2506_21411_amd as dchag

from .test_gpu_attend import LOG, Problem, dev

pytestmark = pytest.mark.gpu

CASES = [
    dict(dtype="bf16", heads=2, kv=2, d=64, ql=[300, 50], borders=LOG),
    dict(dtype="bf16", heads=2, kv=1, d=128, ql=[300, 257], borders=LOG, causal=True),
    dict(dtype="bf16", heads=32, kv=32, d=128, ql=[1100], borders=[1, 40]),
    dict(dtype="bf16", heads=32, kv=8, d=64, ql=[1100, 1030], borders=[1, 2, 70, 300]),
    dict(dtype="f32", heads=2, kv=2, d=64, ql=[300, 50], borders=LOG),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_same_gradients_with_and_without_the_bias_gradient(case):
    p = Problem(seed=53, tail=0, **case)
    q, k, v, dout, kw, qs, ks = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda(), p.kw(), dev(p.qs), dev(p.ks)
    out, lse = dchag.dchag_attend(q, k, v, qs, ks, **kw)
    with_it = dchag.dchag_attend_backward(q, k, v, out, lse, dout, qs, ks, **kw)
    without = dchag.dchag_attend_backward(q, k, v, out, lse, dout, qs, ks, want_dbias=False, **kw)
    assert without[3] is None
    for name, a, b in zip(("dq", "dk", "dv"), with_it, without):
        assert torch.equal(a, b), name
