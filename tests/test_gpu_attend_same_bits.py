"""Two runs of a call give the same bits, on one stream or on two: outputs and every gradient."""
import pytest
import torch

from .test_gpu_attend import LOG, Problem, say

pytestmark = pytest.mark.gpu

CASES = [
    dict(dtype="bf16", heads=4, kv=2, d=64, ql=[150, 70], causal=True, borders=LOG),
    dict(dtype="bf16", heads=8, kv=2, d=128, ql=[1, 1], kl=[4000, 1000], borders=LOG),
    dict(dtype="bf16", heads=16, kv=16, d=64, ql=[129, 257, 1, 190] * 9, borders=LOG),
    dict(dtype="bf16", heads=32, kv=32, d=128, ql=[1030, 1100], borders=LOG),
    dict(dtype="f32", heads=16, kv=8, d=64, ql=[129, 257, 1, 190] * 5, borders=LOG),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_same_bits(case):
    say(f"same bits {case}")
    p = Problem(seed=54, **case)
    one, again = p.run(), p.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = p.run()
    side.synchronize()
    whole = {torch.bfloat16: torch.int16, torch.float32: torch.int32}
    for name, t in one.items():
        bits = lambda x: x.view(whole[x.dtype])  # noqa: E731
        assert torch.equal(bits(t), bits(again[name])), name
        assert torch.equal(bits(t), bits(two[name])), name
