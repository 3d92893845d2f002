"""The operators of the spatial block behind the aggregation, case by case: attention over packed sequences of patch tokens (with
grouped heads, causal or not, with or without a learned relative position bias), its training step, and checkpoints of
activations in 8 bits with the weight gradient that reads them.

  op            entry points                                     who makes it
  attend        dchag_attend                                     inference: whole images or prompts, or single tokens against a cache
  train         dchag_attend + dchag_attend_backward             a training step of the attention: output and every gradient
  checkpoint    dchag_pack8 + dchag_unpack8                      activations put away after the forward pass and fetched for the backward
  weight_grad   dchag_weight_grad8                               weight and bias gradient of a linear layer whose input was put away

`run` makes these calls where `own` is true; otherwise it evaluates the definitions with elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _attend(name, op, dtype, heads, kv_heads, d, q_lens, k_lens, causal=False, borders="", used="", fused=False):
    """q_lens, k_lens: lengths of the sequences ("135x4,77": four of 135 and one of 77); used: how many of a sequence's key rows
    count (a cache with room to grow); borders: distances at which a new bucket of the bias begins; fused: q, k, v are columns of one tensor."""
    c = {"op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "d": d, "q_lens": q_lens, "k_lens": k_lens,
         "causal": causal, "borders": borders, "used": used, "fused": fused}
    return {"name": name, **c} if name else c


def _rows(name, op, dtype, rows, d_in, d_out=0):
    c = {"op": op, "dtype": dtype, "rows": rows, "d_in": d_in, "d_out": d_out}
    return {"name": name, **c} if name else c


#: 16 buckets a side: eight distances of their own, then eight that widen up to 128
LOG16 = "1,2,3,4,5,6,7,8,12,16,23,32,46,64,91"


def listed():
    return [
        # one forecast step of a small model: a token for each of 4 runs against a short history; launches and latency decide
        _attend("step_small_bf16", "attend", "bf16", 8, 8, 32, "1x4", "512x4", causal=True, used="128,77,300,1"),
        # the same for a large model with long histories of different lengths: bound by reading the cache
        _attend("step_long_bf16", "attend", "bf16", 32, 8, 128, "1x16", "16384x16", causal=True, borders=LOG16,
                used="16384,9001,12288,300,8192,4096,16000,5000,10000,777,14001,16384,2048,6000,11111,15000"),
        # the patches of two weather fields (D 1024, 16 heads), each patch sees the whole field, with the relative bias
        _attend("weather_bias_bf16", "attend", "bf16", 16, 16, 64, "2048x2", "2048x2", borders=LOG16),
        # images of different sizes packed one behind the other, odd patch counts
        _attend("images_ragged_bf16", "attend", "bf16", 16, 16, 64, "1024,135,577,256,2048,77,1500,961", "1024,135,577,256,2048,77,1500,961"),
        # a long causal history answered at once by a wide model with grouped heads: the largest forward call
        _attend("history_causal_bf16", "attend", "bf16", 32, 8, 128, "8192", "8192", causal=True),
        # single precision, as one validates: the patches of one weather field, D 512, 8 heads
        _attend("weather_f32_train", "train", "f32", 8, 8, 64, "512x2", "512x2", borders=LOG16),
        # one training step on the headline shape's patches (4 images of 256, D 1024, 16 heads) with the relative bias
        _attend("bands_bias_bf16_train", "train", "bf16", 16, 16, 64, "256x4", "256x4", borders=LOG16),
        # one training step on the wide embedding's grid: 2048 patches, D 4096, 32 heads of 128, with the relative bias
        _attend("wide_bias_bf16_train", "train", "bf16", 32, 32, 128, "2048", "2048", borders=LOG16),
        # packed causal sequences of odd lengths, grouped heads: the largest call
        _attend("packed_causal_bf16_train", "train", "bf16", 32, 8, 128, "4096,3001,777,2500", "4096,3001,777,2500", causal=True, fused=True),
        # the channel tokens of the headline shape put away and fetched: 4 x 512 x 256 tokens of 1024
        _rows("bands_tokens_checkpoint", "checkpoint", "bf16", 524288, 1024),
        # query, key and value projection of grouped heads on 16 images of 2048 patches, D 1024
        _rows("projection_bf16_grad", "weight_grad", "bf16", 32768, 1024, 1536),
        # the same of a small model in single precision, odd sizes: 270 patches, D 384
        _rows("ragged_f32_grad", "weight_grad", "f32", 270, 384, 1152),
    ]


def _lens(text):
    out = []
    for part in text.split(","):
        n, _, times = part.partition("x")
        out += [int(n)] * (int(times) if times else 1)
    return out


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _borders(rng):
    n, r, out = rng.randint(1, 24), 1, []
    for _ in range(n):
        out.append(r)
        r += 1 if rng.random() < 0.5 else rng.randint(1, max(1, r))
        if r > 1000:
            break
    return ",".join(map(str, out))


def draw(rng):
    while True:
        case = _draw(rng)
        cost = work(case)
        if cost["bytes"] < 3.2e9 and cost["flops"] < 9e11:         # no more than the largest listed ones
            return case


def _draw(rng):
    op = rng.choice(["step", "attend", "attend", "train", "train", "checkpoint", "weight_grad"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "checkpoint":
        d = 8 * rng.randint(1, 256)
        return _rows("", op, dtype, _log_int(rng, 1, 400_000_000 // d), d)
    if op == "weight_grad":
        d_in, d_out = 8 * _log_int(rng, 1, 160), 8 * _log_int(rng, 1, 160)
        return _rows("", op, dtype, _log_int(rng, 1, min(32768, 30_000_000_000 // (d_in * d_out))), d_in, d_out)
    d = rng.choice([32, 64, 64, 128, 128, 8 * rng.randint(1, 16)])
    kv = rng.choice([1, 2, 4, 8, 3])
    heads = kv * rng.choice([1, 1, 2, 4])
    borders = _borders(rng) if rng.random() < 0.5 else ""
    if op == "step":
        s = rng.randint(1, 24)
        cap, n = _log_int(rng, 16, 12288), rng.choice([1, 1, 1, 2, 5])
        used = ",".join(str(rng.randint(n, cap)) for _ in range(s))
        return _attend("", "attend", dtype, heads, kv, d, f"{n}x{s}", f"{cap}x{s}", True, borders, used)
    s = rng.choice([1, 2, 3, 5, 8])
    top = _log_int(rng, 16, 3500 if op == "attend" else 1800)
    lens = [max(1, int(top * rng.uniform(0.2, 1.0))) for _ in range(s)]
    text = ",".join(map(str, lens))
    return _attend("", op, dtype, heads, kv, d, text, text, rng.random() < 0.5, borders, "", rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 31))
    return g


def _pack8_plain(x):
    """Codes (e4m3) and exponents (value 2^(byte - 127)) of blocks of 32 of each row."""
    rows, d = x.shape
    blocks = (d + 31) // 32
    y = torch.nn.functional.pad(x.float(), (0, blocks * 32 - d)).view(rows, blocks, 32)
    fin = torch.isfinite(y)
    amax = torch.where(fin, y.abs(), torch.zeros_like(y)).amax(-1)
    man, ex = torch.frexp(amax)                                    # amax = man 2^ex, man in [0.5, 1)
    e = torch.where(amax > 0, ex - 9 + (man > 0.875).int(), torch.full_like(ex, -127)).clamp(min=-127)
    z = torch.where(fin, torch.ldexp(y, -e[..., None].float()), torch.full_like(y, float("nan")))
    return z.to(torch.float8_e4m3fn).view(torch.uint8).view(rows, blocks * 32)[:, :d].contiguous(), (e + 127).to(torch.uint8)


def _unpack8_plain(codes, scales):
    rows, d = codes.shape
    blocks = scales.shape[1]
    y = torch.nn.functional.pad(codes, (0, blocks * 32 - d)).view(torch.float8_e4m3fn).float().view(rows, blocks, 32)
    return torch.ldexp(y, (scales.float() - 127)[..., None]).view(rows, blocks * 32)[:, :d]


def prepare(case, seed):
    g = _gen(seed)
    t = TDT[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(t)

    if case["op"] in ("checkpoint", "weight_grad"):
        rows, d_in = case["rows"], case["d_in"]
        # activations: rows of different size, a few columns much larger than the rest
        x = torch.randn((rows, d_in), generator=g, device="cuda")
        x.mul_(torch.exp(0.5 * torch.randn((rows, 1), generator=g, device="cuda")))
        x.mul_(torch.exp(torch.randn((1, d_in), generator=g, device="cuda")))
        x = x.to(t)
        if case["op"] == "checkpoint":
            return {"case": case, "x": x}
        codes, scales = _pack8_plain(x)
        return {"case": case, "dy": normal(rows, case["d_out"], scale=0.1), "codes": codes, "scales": scales}

    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    ql, kl = _lens(case["q_lens"]), _lens(case["k_lens"])
    tq, tk = sum(ql), sum(kl)
    if case["fused"]:                                              # one projection made them: columns of one tensor
        qkv = normal(tq, (h + 2 * hk) * d)
        q, k, v = qkv[:, :h * d].view(tq, h, d), qkv[:, h * d:(h + hk) * d].view(tk, hk, d), qkv[:, (h + hk) * d:].view(tk, hk, d)
    else:
        q, k, v = normal(tq, h, d), normal(tk, hk, d), normal(tk, hk, d)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    run_sum = lambda a: [sum(a[:i]) for i in range(len(a) + 1)]        # noqa: E731
    borders = [int(b) for b in case["borders"].split(",")] if case["borders"] else None
    nb = (len(borders) + 1) * (1 if case["causal"] else 2) if borders else 0
    st = {"case": case, "q": q, "k": k, "v": v, "q_starts": dev(run_sum(ql)), "k_starts": dev(run_sum(kl)),
          "k_used": dev(_lens(case["used"])) if case["used"] else None, "max_q": max(ql), "max_k": max(kl),
          "borders": borders, "borders_at": dev(borders) if borders else None, "bias": normal(h, nb) if borders else None}
    if case["op"] == "train":
        st["dout"] = normal(tq, h, d)
    return st


# ---------------------------------------------------------------- the passes

class _Padded:
    """The sequences side by side, each padded to the longest: [S, heads, rows, d] in 32 bits, and what may see what."""

    def __init__(self, st):
        c = st["case"]
        self.c, self.st = c, st
        self.h, self.hk, self.d = c["heads"], c["kv_heads"], c["d"]
        self.lq, self.lk = st["max_q"], st["max_k"]
        qs, ks = st["q_starts"].long(), st["k_starts"].long()
        self.nq = qs[1:] - qs[:-1]
        self.nk = ks[1:] - ks[:-1] if st["k_used"] is None else st["k_used"].long()
        dev = st["q"].device
        i, j = torch.arange(self.lq, device=dev), torch.arange(self.lk, device=dev)
        self.q_at = (qs[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
        self.k_at = (ks[:-1, None] + j).clamp(max=st["k"].shape[0] - 1)
        self.q_in, self.k_in = i < self.nq[:, None], j < self.nk[:, None]
        self.off = self.nk - self.nq
        # of each packed row, its place among the padded ones
        row = torch.arange(st["q"].shape[0], device=dev)
        seq = torch.bucketize(row, qs[1:], right=True)
        self.q_back = seq * self.lq + row - qs[seq]
        row = torch.arange(st["k"].shape[0], device=dev)
        seq = torch.bucketize(row, ks[1:], right=True)
        self.k_back = seq * self.lk + row - ks[seq]

    def queries(self, x):
        return (x.float()[self.q_at] * self.q_in[..., None, None]).transpose(1, 2).contiguous()

    def keys(self, x):
        y = (x.float()[self.k_at] * self.k_in[..., None, None]).transpose(1, 2)
        return y.repeat_interleave(self.h // self.hk, 1).contiguous()

    def scores(self, q, k):
        c, st = self.c, self.st
        s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1 / math.sqrt(self.d))
        r = torch.arange(self.lk, device=q.device) - torch.arange(self.lq, device=q.device)[:, None] - self.off[:, None, None]
        if st["bias"] is not None:
            s = s + st["bias"].float()[:, self.bucket(r)].transpose(0, 1)
        ok = self.k_in[:, None, :] & self.q_in[:, :, None]
        if c["causal"]:
            ok = ok & (r <= 0)
        return torch.where(ok[:, None], s, torch.full((), -math.inf, device=q.device))

    def bucket(self, r):
        b = self.st["borders_at"]
        n = torch.bucketize(r.abs(), b, right=True)
        return torch.where(r > 0, n + len(b) + 1, n) if not self.c["causal"] else n.clamp(max=len(b))

    def softmax(self, s):
        m = s.amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp(s - m)
        total = p.sum(-1, keepdim=True)
        return p / total.clamp(min=1e-37), (m + torch.log(total)).squeeze(-1)

    def back_q(self, x):
        return x.transpose(1, 2).flatten(0, 1)[self.q_back]

    def back_k(self, x):
        s, _, lk, d = x.shape
        return x.view(s, self.hk, self.h // self.hk, lk, d).sum(2).transpose(1, 2).flatten(0, 1)[self.k_back]

    def diagonals(self, ds):
        """Sums of ds over the pairs of each bucket."""
        s, h, lq, lk = ds.shape
        x = torch.nn.functional.pad(ds.flip(2), (0, lq)).view(s, h, lq * (lk + lq))[..., :lq * (lk + lq - 1)]
        sums = x.view(s, h, lq, lk + lq - 1).sum(2, dtype=torch.float64)            # by j - i + lq - 1
        r = torch.arange(lk + lq - 1, device=ds.device) - (lq - 1) - self.off[:, None]
        at = self.bucket(r)[:, None].expand(s, h, -1).transpose(0, 1).reshape(h, -1)
        return torch.zeros(self.st["bias"].shape, dtype=torch.float64, device=ds.device).scatter_add_(1, at, sums.transpose(0, 1).reshape(h, -1))


def _plain_attend(st):
    p = _Padded(st)
    q, k, v = p.queries(st["q"]), p.keys(st["k"]), p.keys(st["v"])
    w, lse = p.softmax(p.scores(q, k))
    out = p.back_q(torch.matmul(w, v)).to(st["q"].dtype)
    res = {"out": out, "lse": lse.transpose(0, 1).flatten(1)[:, p.q_back]}
    if p.c["op"] == "attend":
        return res
    scale = 1 / math.sqrt(p.d)
    do = p.queries(st["dout"])
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = w * (dp - (w * dp).sum(-1, keepdim=True))
    t = st["q"].dtype
    res["dq"] = (p.back_q(torch.matmul(ds, k)) * scale).to(t)
    res["dk"] = (p.back_k(torch.matmul(ds.transpose(2, 3).contiguous(), q)) * scale).to(t)
    res["dv"] = p.back_k(torch.matmul(w.transpose(2, 3).contiguous(), do)).to(t)
    if st["bias"] is not None:
        res["dbias"] = p.diagonals(ds).to(t)
    return res


def _plain(st):
    c = st["case"]
    if c["op"] == "checkpoint":
        return _unpack8_plain(*_pack8_plain(st["x"])).to(st["x"].dtype)
    if c["op"] == "weight_grad":
        dy = st["dy"].float()
        x = _unpack8_plain(st["codes"], st["scales"])
        return {"dW": torch.matmul(dy.t(), x).to(st["dy"].dtype), "db": dy.sum(0).to(st["dy"].dtype)}
    return _plain_attend(st)


def _own(st):
    import paper_2506_21411_amd as dchag

    c = st["case"]
    if c["op"] == "checkpoint":
        codes, scales = dchag.dchag_pack8(st["x"])
        return dchag.dchag_unpack8(codes, scales, st["x"].dtype)
    if c["op"] == "weight_grad":
        dW, db = dchag.dchag_weight_grad8(st["dy"], st["codes"], st["scales"])
        return {"dW": dW, "db": db}
    kw = dict(causal=c["causal"], k_used=st["k_used"], bias=st["bias"], borders=st["borders"])
    out, lse = dchag.dchag_attend(st["q"], st["k"], st["v"], st["q_starts"], st["k_starts"], **kw)
    res = {"out": out, "lse": lse}
    if c["op"] == "train":
        dq, dk, dv, dbias = dchag.dchag_attend_backward(st["q"], st["k"], st["v"], out, lse, st["dout"], st["q_starts"], st["k_starts"], **kw)
        res.update(dq=dq, dk=dk, dv=dv)
        if dbias is not None:
            res["dbias"] = dbias
    return res


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "checkpoint":
        n = case["rows"] * case["d_in"]
        held = n + case["rows"] * ((case["d_in"] + 31) // 32)
        return {"bytes": 2 * (n * es + held), "flops": 4 * n}
    if case["op"] == "weight_grad":
        r, i, o = case["rows"], case["d_in"], case["d_out"]
        return {"bytes": r * (i + (i + 31) // 32) + r * o * es + (i * o + o) * es, "flops": 2 * r * i * o}
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    ql = _lens(case["q_lens"])
    kl = _lens(case["used"] or case["k_lens"])
    pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(ql, kl))
    tq, tk = sum(ql), sum(kl)
    moved = (2 * tq * h + 2 * tk * hk) * d * es + 4 * tq * h                        # q, out, k, v, lse
    if case["op"] == "attend":
        return {"bytes": moved, "flops": 4 * d * h * pairs}
    moved += (2 * tq * h + 2 * tk * hk) * d * es                                    # dout, dq, dk, dv
    return {"bytes": moved, "flops": 14 * d * h * pairs}


def _pairs(nq, nk, causal):
    """Pairs that may see each other: the queries are the last nq positions of the nk keys."""
    if not causal:
        return nq * nk
    return sum(max(0, min(nk, nk - nq + i + 1)) for i in range(nq))


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _e4m3_64(y):
    """y rounded to the nearest value of 4 exponent and 3 mantissa bits, ties to even."""
    a = y.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(y) * torch.round(a / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "checkpoint":
        x = st["x"]
        rows, d = x.shape
        out = torch.empty((rows, d), dtype=torch.float64, device=x.device)
        for c0 in range(0, d, 32):                                 # one block of columns at a time
            y = x[:, c0:c0 + 32].double()
            top = y.abs().amax(1, keepdim=True)
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -149) / 448)).clamp(min=-127)
            e = torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e).clamp(min=-127)    # log2 next to a whole number
            e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
            out[:, c0:c0 + 32] = _e4m3_64(y * torch.exp2(-e)) * torch.exp2(e)
        return out
    if case["op"] == "weight_grad":
        dy, code = st["dy"].double(), st["codes"].long()
        man, ex = (code & 7).double(), (code >> 3) & 15
        mag = torch.where(ex > 0, (1 + man / 8) * torch.exp2((ex - 7).double()), man / 8 * 2.0 ** -6)
        x = torch.where(code >= 128, -mag, mag)
        x = x * torch.exp2(st["scales"].double() - 127).repeat_interleave(32, 1)[:, :x.shape[1]]
        return {"dW": torch.matmul(dy.t().contiguous(), x), "db": dy.sum(0)}
    if _cost64(case) > 2e13:
        return None
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    ql, kl = _lens(case["q_lens"]), _lens(case["k_lens"])
    ul = _lens(case["used"]) if case["used"] else kl
    like = lambda x, *shape: torch.zeros(shape or x.shape, dtype=torch.float64, device=x.device)  # noqa: E731
    res = {"out": like(st["q"]), "lse": like(st["q"], h, sum(ql))}
    train = case["op"] == "train"
    if train:
        res.update(dq=like(st["q"]), dk=like(st["k"]), dv=like(st["v"]))
        if st["bias"] is not None:
            res["dbias"] = like(st["bias"])
    if st["bias"] is not None:
        far = max(max(ql), max(kl)) + 1
        side = torch.zeros(far, dtype=torch.long, device=st["q"].device)             # bucket of each distance
        for b in st["borders"]:
            side[b:] += 1
    q0 = k0 = 0
    for nq, room, nk in zip(ql, kl, ul):
        r = torch.arange(nk, device=st["q"].device)[None] - (torch.arange(nq, device=st["q"].device)[:, None] + nk - nq)
        if st["bias"] is not None:
            at = side[r.abs().clamp(max=far - 1)]
            if not case["causal"]:
                at = at + (r > 0) * (len(st["borders"]) + 1)
        for a in range(h):
            q, k, v = st["q"][q0:q0 + nq, a].double(), st["k"][k0:k0 + nk, a // (h // hk)].double(), st["v"][k0:k0 + nk, a // (h // hk)].double()
            s = torch.matmul(q, k.t().contiguous()) / math.sqrt(d)
            if st["bias"] is not None:
                s += st["bias"][a].double()[at]
            if case["causal"]:
                s.masked_fill_(r > 0, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            o = torch.matmul(p, v)
            res["out"][q0:q0 + nq, a], res["lse"][a, q0:q0 + nq] = o, lse
            if train:
                do = st["dout"][q0:q0 + nq, a].double()
                ds = p * (torch.matmul(do, v.t().contiguous()) - (do * o).sum(1, keepdim=True))
                res["dq"][q0:q0 + nq, a] = torch.matmul(ds, k) / math.sqrt(d)
                res["dk"][k0:k0 + nk, a // (h // hk)] += torch.matmul(ds.t().contiguous(), q) / math.sqrt(d)
                res["dv"][k0:k0 + nk, a // (h // hk)] += torch.matmul(p.t().contiguous(), do)
                if st["bias"] is not None:
                    n = st["bias"].shape[1]
                    res["dbias"][a] += torch.bincount(at.flatten(), weights=ds.flatten(), minlength=n)
        q0, k0 = q0 + nq, k0 + room
    return res


def _cost64(case):
    """Flops of a pass with nothing left out for what is masked."""
    kl = _lens(case["used"] or case["k_lens"])
    return sum(a * b for a, b in zip(_lens(case["q_lens"]), kl)) * case["heads"] * case["d"] * (14 if case["op"] == "train" else 4)
