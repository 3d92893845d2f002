"""Host side of the spatial operators: refusals before anything is launched, borders, and the tests' own 64-bit forms against library ones."""
import ctypes
import math
import os

import pytest
import torch

import paper_2506_21411_amd as dchag
from paper_2506_21411_amd.binding import _CAttention

from . import spatial_reference as ref

FAKE = 0x10000          # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dchag.library_path()):
        from paper_2506_21411_amd.build import build
        build(verbose=False)
    return dchag.load_library()


def att(borders=None, **over):
    a = _CAttention()
    a.heads, a.kv_heads, a.head_dim, a.causal, a.sequences, a.rows_q, a.rows_k = 4, 2, 64, 0, 2, 100, 100
    a.q_starts = a.k_starts = FAKE
    if borders is not None:
        a.bias, a.n_borders = FAKE, len(borders)
        a.held = (ctypes.c_int32 * max(1, len(borders)))(*borders)
        a.borders = ctypes.cast(a.held, ctypes.c_void_p)
    for n, v in over.items():
        setattr(a, n, v)
    return a


BAD = [
    (dict(q_starts=None), -1), (dict(k_starts=None), -1), (dict(kv_heads=3), -2), (dict(kv_heads=0), -2), (dict(heads=0), -2),
    (dict(head_dim=136), -2), (dict(head_dim=12), -2), (dict(head_dim=0), -2), (dict(sequences=-1), -2), (dict(rows_q=-1), -2),
    (dict(rows_k=-5), -2), (dict(causal=2), -2), (dict(scale=-1.0), -2), (dict(scale=math.inf), -2), (dict(scale=math.nan), -2),
    (dict(ld_q=248), -2), (dict(ld_q=260), -2), (dict(ld_k=120), -2), (dict(ld_dv=(1 << 23) + 8), -2), (dict(ld_out=-256), -2),
    (dict(q_starts=FAKE + 2), -6), (dict(k_used=FAKE + 1), -6),
    (dict(borders=[]), -2), (dict(borders=[0, 1]), -2), (dict(borders=[2, 2]), -2), (dict(borders=[5, 4]), -2), (dict(borders=[1, 1025]), -2),
    (dict(borders=list(range(1, 65))), -2), (dict(bias=FAKE), -1), (dict(borders=[1], bias=FAKE + 2), -6),
]


@pytest.mark.parametrize("kw,status", BAD, ids=[str(i) for i in range(len(BAD))])
def test_attention_shapes_refused(lib, kw, status):
    a = ctypes.byref(att(**kw))
    assert lib.dchag_attend(1, a, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == status
    assert lib.dchag_attend_backward(1, a, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 40, None) == status
    assert lib.dchag_attend_workspace_bytes(1, a, 0) == 0 == lib.dchag_attend_workspace_bytes(1, a, 1)


def test_attention_pointers_refused(lib):
    a = ctypes.byref(att())
    good = [FAKE] * 6 + [1 << 40, None]
    assert lib.dchag_attend(7, a, *good) == -3
    assert lib.dchag_attend(1, None, *good) == -1
    for i in range(5):
        assert lib.dchag_attend(1, a, *good[:i], None, *good[i + 1:]) == -1
        assert lib.dchag_attend(1, a, *good[:i], FAKE + 4, *good[i + 1:]) == -6
    assert lib.dchag_attend(1, a, *good[:5], None, *good[6:]) == -4
    assert lib.dchag_attend(1, a, *good[:5], FAKE + 16, *good[6:]) == -4
    assert lib.dchag_attend(1, a, *good[:6], 16, None) == -4
    good = [FAKE] * 9 + [None, FAKE, 1 << 40, None]
    for i in range(9):
        assert lib.dchag_attend_backward(1, a, *good[:i], None, *good[i + 1:]) == -1
        assert lib.dchag_attend_backward(1, a, *good[:i], FAKE + 4, *good[i + 1:]) == -6
    assert lib.dchag_attend_backward(1, a, *good[:9], FAKE, *good[10:]) == -2          # dbias without a bias
    assert lib.dchag_attend_backward(1, a, *good[:11], 16, None) == -4
    assert lib.dchag_attend_workspace_bytes(1, a, 2) == 0


def test_calls_too_large_for_a_launch_are_refused(lib):
    a = ctypes.byref(att(heads=4096, kv_heads=4096, head_dim=8, rows_q=2 ** 31 - 1, rows_k=2 ** 31 - 1))
    assert lib.dchag_attend(1, a, *[FAKE] * 6, 1 << 60, None) == -2
    assert lib.dchag_attend_backward(1, a, *[FAKE] * 9, None, FAKE, 1 << 60, None) == -2


def test_keep8_refused(lib):
    for f in (lib.dchag_pack8, lib.dchag_unpack8):
        assert f(7, 4, 64, 0, FAKE, FAKE, FAKE, None) == -3
        for rows, D, ld in ((-1, 64, 0), (4, 60, 0), (4, 0, 0), (4, 64, 56), (4, 64, 68), (4, (1 << 20) + 8, 0), (4, 64, (1 << 23) + 8), (1 << 62, 64, 0)):
            assert f(1, rows, D, ld, FAKE, FAKE, FAKE, None) == -2, (rows, D, ld)
        for i in range(3):
            p = [FAKE] * 3
            p[i] = None
            assert f(1, 4, 64, 0, *p, None) == -1
            p[i] = FAKE + 8
            assert f(1, 4, 64, 0, *p, None) == -6
    g, ws = lib.dchag_weight_grad8, lib.dchag_weight_grad8_workspace_bytes
    assert g(7, 4, 64, 64, 0, *[FAKE] * 6, 1 << 40, None) == -3
    for rows, o, i, ld in ((-1, 64, 64, 0), (4, 12, 64, 0), (4, 64, 4, 0), (4, 64, 64, 56), (4, 64, 64, 65), (4, 1 << 21, 64, 0)):
        assert g(1, rows, o, i, ld, *[FAKE] * 6, 1 << 40, None) == -2
    assert ws(1, -1, 64, 64) == 0 and ws(1, 4, 12, 64) == 0 and ws(9, 4, 64, 64) == 0 and ws(1, 4, 64, 64) > 0
    for i in range(4):
        p = [FAKE] * 5
        p[i] = None
        assert g(1, 4, 64, 64, 0, *p, FAKE, 1 << 40, None) == -1
    for i in range(5):
        p = [FAKE] * 5
        p[i] = FAKE + 2
        assert g(1, 4, 64, 64, 0, *p, FAKE, 1 << 40, None) == -6
    assert g(1, 100000, 64, 64, 0, *[FAKE] * 5, FAKE, 16, None) == -4
    assert g(1, 4, 64, 64, 0, *[FAKE] * 5, None, 1 << 40, None) == -4


def test_binding_refuses_what_the_library_cannot_see():
    q, k = torch.zeros(6, 4, 64), torch.zeros(6, 2, 64)
    s = torch.zeros(2, dtype=torch.int32)
    for args, kw in (((q[0], k, k, s, s), {}), ((q, k, k[:5], s, s), {}), ((q, k[..., :32], k[..., :32], s, s), {}),
                     ((q.transpose(0, 1), k, k, s, s), {}), ((q[:1].expand(6, 4, 64), k, k, s, s), {}), ((q, k, k, s, s[:1]), {}), ((q, k, k, s[None], s), {}),
                     ((q, k, k, s, s), dict(bias=torch.zeros(4, 4))), ((q, k, k, s, s), dict(borders=[1])),
                     ((q, k, k, s, s), dict(bias=torch.zeros(4, 3), borders=[1])), ((q, k, k, s, s), {})):   # the last: not on a device
        with pytest.raises(ValueError):
            dchag.dchag_attend(*args, **kw)
    with pytest.raises(ValueError):
        dchag.dchag_pack8(torch.zeros(4, 8, 2))
    with pytest.raises(ValueError):
        dchag.dchag_pack8(torch.zeros(8, 8).t()[:, ::2])
    with pytest.raises(ValueError):
        dchag.dchag_pack8(torch.zeros(1, 8).expand(4, 8))
    with pytest.raises(ValueError):
        dchag.dchag_weight_grad8(torch.zeros(4, 8), torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.uint8))


def test_log_borders():
    assert dchag.log_borders(2, 5) == [1]
    assert dchag.log_borders(16, 128) == [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]   # 8 * 16^(k/8), rounded up; 16, 32, 64 exactly
    for buckets in (2, 3, 8, 32, 64):
        b = dchag.log_borders(buckets, 1024)
        assert len(b) == buckets - 1 and all(x < y for x, y in zip(b, b[1:])) and b[-1] < 1024
    with pytest.raises(ValueError):
        dchag.log_borders(1, 10)
    with pytest.raises(ValueError):
        dchag.log_borders(8, 4)


@pytest.mark.parametrize("causal", [False, True])
def test_reference_against_the_library(causal):
    """The 64-bit form the GPU tests use, against torch's attention with an additive mask and its gradients."""
    gen = torch.Generator().manual_seed(1)
    h, hk, d, ql, kl, borders = 4, 2, 16, [5, 9], [7, 9], [1, 2, 4]
    qs, ks = [0, 5, 14], [0, 7, 16]
    r = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    q, k, v, bias, dout = r(14, h, d), r(16, hk, d), r(16, hk, d), r(h, 4 * (1 if causal else 2)), r(14, h, d)
    want = ref.attention(q, k, v, qs, ks, causal, 0.0, None, bias, borders, dout)
    leaves = [x.clone().requires_grad_() for x in (q, k, v, bias)]
    outs = []
    for s in range(2):
        Q, K, V = leaves[0][qs[s]:qs[s + 1]], leaves[1][ks[s]:ks[s + 1]], leaves[2][ks[s]:ks[s + 1]]
        rel = torch.arange(kl[s])[None] - (torch.arange(ql[s])[:, None] + kl[s] - ql[s])
        mask = leaves[3][:, ref.bucket(rel, borders, causal)]
        if causal:
            mask = mask.masked_fill(rel > 0, -math.inf)
        outs.append(torch.nn.functional.scaled_dot_product_attention(Q.transpose(0, 1), K.transpose(0, 1).repeat_interleave(h // hk, 0),
                                                                     V.transpose(0, 1).repeat_interleave(h // hk, 0), attn_mask=mask).transpose(0, 1))
    out = torch.cat(outs)
    out.backward(dout)
    assert torch.allclose(want["out"][0], out.detach(), atol=1e-12)
    for n, leaf in zip(("dq", "dk", "dv", "dbias"), leaves):
        assert torch.allclose(want[n][0], leaf.grad, atol=1e-12), n


def test_reference_of_8_bits_against_the_library():
    """Codes of the format's definition against torch's e4m3 conversion, on every value of a grid with all its ties."""
    x = torch.cat([torch.linspace(-448, 448, 28673), torch.linspace(-0.05, 0.05, 20481)])
    x = torch.nn.functional.pad(x, (0, -x.numel() % 8)).view(-1, 8)
    x = torch.cat([x, torch.full((x.shape[0], 24), 448.0)], 1)         # exponent 127 everywhere
    values, codes, held = ref.pack8(x)
    assert bool((held == 127).all())
    lib = x.to(torch.float8_e4m3fn)
    assert torch.equal(lib.double(), values)
    assert torch.equal(lib.view(torch.uint8)[values != 0], codes[values != 0])
