"""Causal rows that see no key, with a gradient that is not finite at their outputs: dq there is 0, and nothing else has a part of it."""
import pytest
import torch

from .test_gpu_attend import LOG, Problem, say

pytestmark = pytest.mark.gpu

CASES = [
    # rows that see nothing and rows that see keys in one wavefront; the last two: more than two tiles of keys for the first rows' workgroup
    dict(dtype="f32", heads=2, kv=1, d=64, ql=[200, 40], kl=[150, 0], borders=LOG),
    dict(dtype="f32", heads=2, kv=2, d=32, ql=[130], kl=[125]),
    dict(dtype="f32", heads=16, kv=16, d=64, ql=[1030], kl=[1000], borders=[1, 2, 40]),
    dict(dtype="bf16", heads=4, kv=2, d=64, ql=[200, 40], kl=[150, 0], borders=LOG),
    dict(dtype="bf16", heads=32, kv=32, d=128, ql=[1100], kl=[1073], borders=[1, 2, 40]),
    dict(dtype="bf16", heads=32, kv=32, d=64, ql=[1100], kl=[1073]),
]


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_gradients_of_rows_that_see_nothing(case, value):
    say(f"blind rows {case} {value}")
    p = Problem(causal=True, seed=51, tail=2, **case)
    want = p.want()
    q0 = 0
    for nq, nk in zip(case["ql"], case["kl"]):
        p.dout[q0:q0 + max(0, nq - nk)] = value
        q0 += nq
    p.check(want=want)
