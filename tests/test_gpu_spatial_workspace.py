"""A workspace of one's own: of any type, but on the device and in one piece; others are refused before anything is launched."""
import pytest
import torch

import paper_2506_21411_amd as dchag

from .test_gpu_attend import Problem, dev

pytestmark = pytest.mark.gpu


def calls():
    """Of each call with a workspace: a function that makes it, and its results without one."""
    p = Problem("bf16", 4, 2, 64, [70, 30], causal=True, seed=55, tail=0)
    q, k, v, dout, at = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda(), (dev(p.qs), dev(p.ks))
    x, dy = torch.randn(1000, 64, device="cuda"), torch.randn(1000, 32, device="cuda")
    codes, scales = dchag.dchag_pack8(x)
    out, lse = dchag.dchag_attend(q, k, v, *at, causal=True)
    return [lambda ws: dchag.dchag_attend(q, k, v, *at, causal=True, workspace=ws),
            lambda ws: dchag.dchag_attend_backward(q, k, v, out, lse, dout, *at, causal=True, workspace=ws)[:3],
            lambda ws: dchag.dchag_weight_grad8(dy, codes, scales, workspace=ws)]


@pytest.mark.parametrize("which", range(3))
def test_workspace_of_ones_own(which):
    call = calls()[which]
    want = call(None)
    for ws in (torch.empty(1 << 22, dtype=torch.uint8, device="cuda"), torch.empty(1 << 20, device="cuda")):
        for a, b in zip(call(ws), want):
            assert torch.equal(a, b)
    for ws in (torch.empty(1 << 22, dtype=torch.uint8), torch.empty(1 << 23, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(ws)
    with pytest.raises(dchag.DchagError):
        call(torch.empty(16, dtype=torch.uint8, device="cuda"))
