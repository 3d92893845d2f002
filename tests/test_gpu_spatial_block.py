"""The operators as they are used together: the aggregation's tokens are put away in 8 bits, projected to queries, keys and values, attended to
with the relative bias, and a training step's backward pass goes the same way back, reading the 8 bits; all gradients against 64-bit autograd."""
import math

import pytest
import torch

import paper_2506_21411_amd as dchag

from . import spatial_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 2e-2)])
def test_training_step_of_a_spatial_block(dtype, tol):
    """Images of 40 patches by one call of the aggregation, then a packed batch of them: one whole, one cropped to 23 patches."""
    B, C, H, W, p, D, heads, kv = 2, 6, 20, 32, 4, 128, 4, 2
    N, d = (H // p) * (W // p), D // heads
    gen = torch.Generator().manual_seed(1)
    r = lambda *s, scale=1.0: (torch.randn(s, generator=gen) * scale).to(dtype).cuda()  # noqa: E731
    levels = [dchag.LevelWeights(g, r(n, D), *[r(n, D, D, scale=D ** -0.5) for _ in range(4)]) for n, g in ((2, 3), (1, 2))]
    tokens = dchag.dchag_forward(r(B, C, H, W), r(C, D, p * p, scale=1 / p), None, None, levels, p, 4)
    lens = [N, 23]
    x = torch.cat([tokens[0], tokens[1, :23]])
    rows, width = x.shape[0], (heads + 2 * kv) * d
    Wqkv, Wo = r(width, D, scale=2 * D ** -0.5), r(D, D, scale=D ** -0.5)
    borders = dchag.log_borders(4, 16)
    bias, dy = r(heads, 8), r(rows, D)
    starts = torch.tensor([0, N, N + 23], dtype=torch.int32, device="cuda")

    # forward: what is kept is the 8-bit input, q, k, v, out and lse
    codes, scales = dchag.dchag_pack8(x)
    qkv = dchag.dchag_unpack8(codes, scales, dtype) @ Wqkv.t()
    cut = lambda t: (t[:, :D].view(rows, heads, d), t[:, D:D + kv * d].view(rows, kv, d), t[:, D + kv * d:].view(rows, kv, d))  # noqa: E731
    q, k, v = cut(qkv)
    kw = dict(bias=bias, borders=borders)
    out, lse = dchag.dchag_attend(q, k, v, starts, starts, **kw)
    y = out.view(rows, D) @ Wo.t()
    # backward
    dout = (dy @ Wo).view(rows, heads, d)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = cut(dqkv)
    _, _, _, dbias = dchag.dchag_attend_backward(q, k, v, out, lse, dout, starts, starts, dq=dq, dk=dk, dv=dv, **kw)
    dW, db = dchag.dchag_weight_grad8(dqkv, codes, scales)
    dx = dqkv @ Wqkv

    leaves = [t.double().cpu().requires_grad_() for t in (Wqkv, bias, torch.zeros(width), torch.zeros(0))]
    x8 = ref.pack8(x.cpu())[0].requires_grad_()
    Q, K, V = cut(x8 @ leaves[0].t() + leaves[2])
    parts = []
    for s, n in zip((0, N), lens):
        rel = torch.arange(n)[None] - torch.arange(n)[:, None]
        sc = torch.einsum("iad,jad->aij", Q[s:s + n], K[s:s + n].repeat_interleave(heads // kv, 1)) / math.sqrt(d)
        w = torch.softmax(sc + leaves[1][:, ref.bucket(rel, borders, False)], -1)
        parts.append(torch.einsum("aij,jad->iad", w, V[s:s + n].repeat_interleave(heads // kv, 1)))
    want = torch.cat(parts).reshape(rows, D) @ Wo.double().cpu().t()
    want.backward(dy.double().cpu())
    pairs = dict(y=(y, want.detach()), dW=(dW, leaves[0].grad), dbias=(dbias, leaves[1].grad), db=(db, leaves[2].grad), dx=(dx, x8.grad))
    for name, (got, exp) in pairs.items():
        off = float((got.double().cpu() - exp).abs().max() / exp.abs().max())
        print(f"{name}: max|err|/max|ref| = {off:.2e}", flush=True)
        assert off < tol, name                                     # the library's measure and bounds for a chain of roundings
