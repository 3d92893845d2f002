"""Plain 64-bit forms of the spatial operators (attention over packed sequences, 8-bit rows) for their tests, with bounds on how far a
kernel may be off.  Everything here is on the CPU, one sequence and one head at a time.

Bounds: a rounding to type t is off by at most u = finfo(t).eps / 2 of the value; fp32 sums of n terms by n 2^-24 of the sum of
magnitudes.  e below bounds the relative error of P that scores off by a few 2^-24 of their terms, the exponential and the sum over the
keys leave; P and dS are rounded to the tensors' type once before they are multiplied (nothing is lost in fp32)."""
from __future__ import annotations

import math

import torch

F32 = 2.0 ** -24


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def bucket(r, borders, causal):
    n = sum((r.abs() >= b).long() for b in borders)
    return n if causal else n + (r > 0) * (len(borders) + 1)


def spans(q_starts, k_starts, k_used=None):
    for s in range(len(q_starts) - 1):
        nk = k_starts[s + 1] - k_starts[s]
        yield q_starts[s], q_starts[s + 1] - q_starts[s], k_starts[s], nk if k_used is None else min(k_used[s], nk)


def attention(q, k, v, q_starts, k_starts, causal=False, scale=0.0, k_used=None, bias=None, borders=None, dout=None):
    """{name: (value, bound)} in 64 bits; rows of no sequence are NaN.  The bounds are for kernels given tensors of q's type."""
    dtype, u = q.dtype, unit(q.dtype)
    r8 = u if dtype != torch.float32 else 0.0                     # rounding of P and dS
    q, k, v = q.double(), k.double(), v.double()
    h, hk, d = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or 1 / math.sqrt(d)
    new = lambda *s: [torch.full(s, float("nan"), dtype=torch.float64), torch.full(s, float("nan"), dtype=torch.float64)]  # noqa: E731
    res = {"out": new(*q.shape), "lse": new(h, q.shape[0])}
    if dout is not None:
        dout = dout.double()
        res.update(dq=new(*q.shape), dk=new(*k.shape), dv=new(*v.shape))
        if bias is not None:
            res["dbias"] = [torch.zeros(bias.shape, dtype=torch.float64), torch.zeros(bias.shape, dtype=torch.float64)]
    for q0, nq, k0, nk in spans(q_starts, k_starts, k_used):
        if dout is not None:
            for n in ("dk", "dv"):
                for t in res[n]:
                    t[k0:k0 + nk] = 0
        r = torch.arange(nk)[None] - (torch.arange(nq)[:, None] + nk - nq)
        seen = r <= 0 if causal else torch.ones_like(r, dtype=torch.bool)
        for a in range(h):
            kv = a * hk // h
            Q, K, V = q[q0:q0 + nq, a], k[k0:k0 + nk, kv], v[k0:k0 + nk, kv]
            terms = scale * Q.abs() @ K.abs().T
            s = scale * Q @ K.T
            ok = seen
            if bias is not None:
                b = bias[a].double()[bucket(r, borders, causal)] if nq and nk else s
                ok = ok & (b > -1e30)
                s = s + torch.where(ok, b, torch.zeros_like(b))
                terms = terms + torch.where(ok, b.abs(), torch.zeros_like(b))
            s = torch.where(ok, s, torch.full_like(s, -math.inf))
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            some = torch.isfinite(lse)
            P = torch.where(ok & some[:, None], torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
            # a visible value that is not finite makes its rows not finite; one that is not visible has no part
            mul = lambda w, x: torch.where(w.ne(0)[:, :, None], w[:, :, None] * x[None], 0.0).sum(1) if not torch.isfinite(x).all() else w @ x  # noqa: E731
            top = terms.max() if terms.numel() and torch.isfinite(terms).all() else torch.tensor(50.0)
            e = 2 * F32 * ((d + 8) * top + nk + 16)
            out = mul(P, V)
            at = (slice(q0, q0 + nq), a)
            res["out"][0][at] = out
            res["out"][1][at] = (r8 + e) * mul(P, V.abs()) + (u + 4 * F32) * out.abs()
            res["lse"][0][a, q0:q0 + nq] = lse
            res["lse"][1][a, q0:q0 + nq] = e + 4 * F32 * torch.where(some, lse.abs(), 0.0)
            if dout is None:
                continue
            G = dout[at]
            dP, size = G @ V.T, G.abs() @ V.abs().T
            delta = (G * out).sum(1, keepdim=True)
            off = (u + e + d * F32) * (G.abs() * (out.abs() + P @ V.abs())).sum(1, keepdim=True)   # of delta: out is rounded
            dS = torch.where(ok, P * (dP - delta), 0.0)
            # a masked pair's P is 0, whatever dP is
            ds_off = torch.where(P > 0, P * (off + (d + 4) * F32 * size) + (e + 4 * F32) * P * (dP.abs() + delta.abs()), 0.0)
            wide = ds_off + r8 * dS.abs()
            res["dq"][0][at] = scale * mul(dS, K)
            res["dq"][1][at] = scale * mul(wide + nk * F32 * dS.abs(), K.abs()) + (u + 4 * F32) * (scale * mul(dS, K)).abs()
            kat = (slice(k0, k0 + nk), kv)
            res["dk"][0][kat] += scale * mul(dS.T, Q)
            res["dk"][1][kat] += scale * mul((wide + nq * F32 * dS.abs()).T, Q.abs())
            res["dv"][0][kat] += mul(P.T, G)
            res["dv"][1][kat] += mul((r8 + e + nq * F32) * P.T, G.abs())
            if bias is not None and nq and nk:
                idx = bucket(r, borders, causal).clamp(max=bias.shape[1] - 1)
                for i, x in enumerate((dS, ds_off + (nq * nk) ** 0.5 * 4 * F32 * dS.abs())):
                    res["dbias"][i][a].index_add_(0, idx.flatten(), x.flatten())
    for n in ("dk", "dv", "dbias"):
        if n in res:
            res[n][1] += (u + 4 * F32) * res[n][0].abs()
    return {n: tuple(x) for n, x in res.items()}


def pack8(x):
    """(values the codes stand for, codes, bytes) of rows x, in 64 bits, from the format's definition."""
    x = x.double()
    rows, d = x.shape
    blocks = (d + 31) // 32
    codes, held = torch.zeros((rows, d), dtype=torch.uint8), torch.zeros((rows, blocks), dtype=torch.uint8)
    values = torch.zeros_like(x)
    for b in range(blocks):
        y = x[:, b * 32:(b + 1) * 32]
        fin = torch.isfinite(y)
        top = torch.where(fin, y.abs(), 0.0).amax(1)
        byte = torch.zeros(rows, dtype=torch.long)
        for _ in range(255):                                       # the smallest byte whose largest number reaches top
            byte += (448.0 * torch.exp2((byte - 127).double()) < top).long()
        sc = torch.exp2((byte - 127).double())[:, None]
        z = torch.where(fin, y, 0.0) / sc
        z = torch.where((byte == 247)[:, None], z.clamp(-240, 240), z)   # 256 * 2^120 is no number of the types
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
        n = torch.round(z.abs() / step)                            # to even
        mag = n * step
        ex = torch.floor(torch.log2(mag.clamp(min=2.0 ** -6)))
        normal = mag >= 2.0 ** -6
        code = torch.where(normal, (ex + 7) * 8 + (mag / torch.exp2(ex) - 1) * 8, mag * 2.0 ** 9).long()
        code = torch.where(torch.signbit(y), code + 128, code)
        codes[:, b * 32:(b + 1) * 32] = torch.where(fin, code, torch.full_like(code, 127)).to(torch.uint8)
        held[:, b] = byte.to(torch.uint8)
        values[:, b * 32:(b + 1) * 32] = torch.where(fin, torch.sign(z) * mag * sc, float("nan"))
    return values, codes, held


def check(name, got, want, bound):
    """Every entry of got within its bound of want; NaN and infinities where want has them."""
    got = got.detach().double().cpu()
    special = ~torch.isfinite(want)
    same = torch.where(want.isnan(), got.isnan(), got == want)
    assert bool(same[special].all()), f"{name}: not finite where it should be finite, or the reverse"
    off = torch.where(special, 0.0, (got - want).abs())
    bad = ~(off <= bound + 1e-30) & ~special
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} entries beyond their bound, first {bad.nonzero()[0].tolist()}: "
                                 f"{got[bad][0]:.6g} for {want[bad][0]:.6g} +- {bound[bad][0]:.3g}")
