"""Starts that decrease: a sequence that would end before it begins is empty, and the others have their results where they lie."""
import pytest
import torch

import paper_2506_21411_amd as dchag

from .test_gpu_attend import Problem, dev

pytestmark = pytest.mark.gpu


# the second half of the rows, an empty sequence back to the first row, the first half; then as many empty sequences as fill the list
@pytest.mark.parametrize("empty", [0, 150], ids=["few sequences", "many sequences"])
@pytest.mark.parametrize("case", [dict(heads=2, kv=1, d=64, ql=[90, 130], kl=[100, 160]), dict(heads=8, kv=2, d=64, ql=[3, 1], kl=[4000, 1500]),
                                  dict(heads=8, kv=8, d=32, ql=[2, 2], kl=[300, 300])], ids=["tiles", "few", "few whole"])
def test_sequences_out_of_order(case, empty):
    p = Problem("bf16", causal=True, seed=56, **case)
    q, k, v, dout = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda()
    turned = lambda starts: dev([starts[1], starts[2], 0, starts[1]] + [starts[1]] * empty)  # noqa: E731
    plain = lambda starts: dev(starts + [starts[2]] * (1 + empty))  # noqa: E731
    got = {}
    for order in (plain, turned):
        qs, ks = order(p.qs), order(p.ks)
        out, lse = dchag.dchag_attend(q, k, v, qs, ks, causal=True, out=torch.full_like(q, 7.0), lse=torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda"))
        got[order] = [out, lse, *dchag.dchag_attend_backward(q, k, v, out, lse, dout, qs, ks, causal=True, dq=torch.full_like(q, 7.0),
                                                            dk=torch.full_like(k, 7.0), dv=torch.full_like(k, 7.0))[:3]]
    for a, b in zip(got[plain], got[turned]):
        assert torch.equal(a, b)
