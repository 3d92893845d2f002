"""The bias gradient of attention in 64 bits with bounds narrow enough that a sum which was lost does not pass for a rounding.

An entry of the bias gradient adds up dS over all pairs of a bucket.  What a kernel's dS is off by is of two kinds, and both are counted by
their variances here, not by their magnitudes (which add up to more than the entries themselves):

* once for a row, off_i in delta_i, which every pair of the row has with weight P_ij: out comes rounded to the type, every column by at
  most u = eps / 2 of itself, evenly spread in the worst case (variance u^2 / 3), and it was formed from weights P that were rounded the same
  way.  So off_i has the variance u^2 / 3 (sum_c do_c^2 out_c^2 + sum_j P_ij^2 dP_ij^2), and a bucket has off_i times the row's P in it;
* once for a pair: scores and dP are fp32 sums of d terms, at most (d + 8) 2^-24 of the terms' magnitudes, the exponential and the sum a few 2^-24.

A row's common factor in P (its lse) changes its part of an entry by that factor.  Entries are bounded by six standard deviations and the rounding
of the result.  In the last bucket of a side the kernels take the row's error out for every tile whose pairs are all in it, so only pairs
nearer than the last border + 128 (where tiles with other buckets end) have it there."""
from __future__ import annotations

import math

import torch

from . import spatial_reference as ref

SIGMAS = 6.0
REACH = 128


def bias_gradient(q, k, v, q_starts, k_starts, bias, borders, dout, causal=False, k_used=None):
    """(dbias, bound, dbias without the pairs beyond the last border) in 64 bits, each [heads, buckets]."""
    dtype = q.dtype
    u = ref.unit(dtype)
    rounded = u if dtype != torch.float32 else 0.0
    h, hk, d = q.shape[1], k.shape[1], q.shape[2]
    scale, n = 1 / math.sqrt(d), bias.shape[1]
    new = lambda: torch.zeros(bias.shape, dtype=torch.float64)  # noqa: E731
    value, var, near = new(), new(), new()
    for q0, nq, k0, nk in ref.spans(q_starts, k_starts, k_used):
        if not nq or not nk:
            continue
        r = torch.arange(nk)[None] - (torch.arange(nq)[:, None] + nk - nq)
        seen = r <= 0 if causal else torch.ones_like(r, dtype=torch.bool)
        at = ref.bucket(r, borders, causal).clamp(max=n - 1)
        far = r.abs() >= borders[-1]
        own = ~(r.abs() >= borders[-1] + REACH)                    # pairs that keep their share of the row's error
        for a in range(h):
            Q, K, V, G = (x.double() for x in (q[q0:q0 + nq, a], k[k0:k0 + nk, a * hk // h], v[k0:k0 + nk, a * hk // h], dout[q0:q0 + nq, a]))
            s = scale * Q @ K.T + bias[a].double()[at]
            terms = scale * Q.abs() @ K.abs().T + bias[a].double()[at].abs()
            s = torch.where(seen, s, torch.full_like(s, -math.inf))
            lse = torch.logsumexp(s, 1, keepdim=True)
            P = torch.where(torch.isfinite(lse) & seen, torch.exp(s - torch.where(torch.isfinite(lse), lse, 0.0)), 0.0)
            out = P @ V
            dP = G @ V.T
            delta = (G * out).sum(1, keepdim=True)
            dS = P * (dP - delta)
            row_var = u ** 2 / 3 * (G * out).square().sum(1, keepdim=True) + rounded ** 2 / 3 * (P * dP).square().sum(1, keepdim=True)
            pair = ref.F32 * ((d + 8) * terms + 8) * dS.abs() + ref.F32 * (d + 8) * P * (G.abs() @ V.abs().T)
            by = lambda x: torch.zeros((nq, n), dtype=torch.float64).scatter_add_(1, at, x)  # noqa: E731
            rows = by(dS)
            common = ref.F32 * (16 + (d + 8) * (P * terms).sum(1, keepdim=True)) * rows   # lse: scores' errors weighed by P
            value[a] += rows.sum(0)
            near[a] += by(torch.where(far, 0.0, dS)).sum(0)
            var[a] += (by(torch.where(own, P, 0.0)).square() * row_var).sum(0) + by(pair.square()).sum(0) + common.square().sum(0)
    return value, SIGMAS * var.sqrt() + (u + 8 * ref.F32) * value.abs(), near
