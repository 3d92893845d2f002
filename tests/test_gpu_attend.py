"""Attention over packed sequences, with grouped heads, causal masks, relative position bias and caches, forward and backward,
against the 64-bit form, entry by entry within derived bounds."""
import itertools

import pytest
import torch

import paper_2506_21411_amd as dchag

from . import spatial_reference as ref

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
LOG = dchag.log_borders(8, 32)


def say(msg):
    print(msg, flush=True)


def starts(lens):
    return list(itertools.accumulate(lens, initial=0))


def dev(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


def normal(gen, dtype, *shape):
    return torch.randn(shape, generator=gen).to(TDT[dtype])


class Problem:
    """Tensors of one call, on the host; `tail` rows behind the last sequence hold NaN."""

    def __init__(self, dtype, heads, kv, d, ql, kl=None, causal=False, borders=None, used=None, seed=0, tail=3, train=True, scale=0.0):
        gen = torch.Generator().manual_seed(seed)
        kl = ql if kl is None else kl
        self.qs, self.ks, self.used, self.causal, self.borders, self.scale = starts(ql), starts(kl), used, causal, borders, scale
        tq, tk = self.qs[-1] + tail, self.ks[-1] + tail
        self.q, self.k, self.v = normal(gen, dtype, tq, heads, d), normal(gen, dtype, tk, kv, d), normal(gen, dtype, tk, kv, d)
        self.dout = normal(gen, dtype, tq, heads, d) if train else None
        self.bias = None
        if borders:
            self.bias = normal(gen, dtype, heads, (len(borders) + 1) * (1 if causal else 2))
        self.in_q, self.in_k = torch.zeros(tq, dtype=torch.bool), torch.zeros(tk, dtype=torch.bool)
        for q0, nq, k0, nk in ref.spans(self.qs, self.ks, used):
            self.in_q[q0:q0 + nq] = True
            self.in_k[k0:k0 + nk] = True
        for t, rows in ((self.q, self.in_q), (self.dout, self.in_q), (self.k, self.in_k), (self.v, self.in_k)):
            if t is not None:
                t[~rows] = float("nan")

    def want(self):
        return ref.attention(self.q, self.k, self.v, self.qs, self.ks, self.causal, self.scale, self.used, self.bias, self.borders, self.dout)

    def kw(self):
        return dict(causal=self.causal, scale=self.scale, k_used=dev(self.used), bias=None if self.bias is None else self.bias.cuda(), borders=self.borders)

    def run(self):
        """Outputs by name; what a call must not write is 7."""
        q, k, v, kw = self.q.cuda(), self.k.cuda(), self.v.cuda(), self.kw()
        sevens = lambda t: torch.full_like(t, 7.0)  # noqa: E731
        lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
        out, lse = dchag.dchag_attend(q, k, v, dev(self.qs), dev(self.ks), out=sevens(q), lse=lse, **kw)
        got = {"out": out, "lse": lse}
        if self.dout is not None:
            dq, dk, dv, db = dchag.dchag_attend_backward(q, k, v, out, lse, self.dout.cuda(), dev(self.qs), dev(self.ks), dq=sevens(q), dk=sevens(k),
                                                         dv=sevens(v), **kw)
            got.update(dq=dq, dk=dk, dv=dv)
            if db is not None:
                got["dbias"] = db
        torch.cuda.synchronize()
        return got

    def check(self, got=None, want=None):
        got, want = got or self.run(), want or self.want()
        for name, (value, bound) in want.items():
            g = got[name]
            rows = self.in_q if name in ("out", "dq", "lse") else self.in_k if name in ("dk", "dv") else None
            if rows is not None:
                left = g[:, ~rows.cuda()] if name == "lse" else g[~rows.cuda()]
                assert bool((left == 7.0).all()), f"{name}: rows of no sequence were written"
                g, value, bound = (x[:, rows.to(x.device)] if name == "lse" else x[rows.to(x.device)] for x in (g, value, bound))
            ref.check(name, g, value, bound)


CASES = [
    # heads, kv, d, ql, kl, causal, borders, used
    dict(heads=2, kv=2, d=64, ql=[1]),
    dict(heads=3, kv=1, d=32, ql=[129, 0, 1, 64, 63, 200]),
    dict(heads=4, kv=2, d=128, ql=[65, 190, 0, 33], causal=True),
    dict(heads=4, kv=4, d=8, ql=[70, 131], causal=True, borders=[1]),
    dict(heads=2, kv=1, d=40, ql=[100, 37, 129], borders=LOG),
    dict(heads=6, kv=2, d=96, ql=[150, 3], borders=[2, 5, 9, 40], causal=True),
    dict(heads=2, kv=2, d=64, ql=[300, 260], borders=[1, 2, 3, 100, 1024]),
    dict(heads=2, kv=2, d=128, ql=[257], borders=[3, 150]),
    # more queries than keys: causal rows that see nothing; no keys at all; fewer queries than keys
    dict(heads=2, kv=1, d=64, ql=[130, 40, 90, 50], kl=[70, 0, 200, 50], causal=True),
    dict(heads=2, kv=1, d=64, ql=[130, 40, 90], kl=[70, 0, 200], borders=LOG),
    dict(heads=2, kv=2, d=32, ql=[80, 70, 40], kl=[100, 90, 64], used=[100, 7, 0], causal=True, borders=LOG),
    dict(heads=2, kv=1, d=64, ql=[90, 130], kl=[200, 130], used=[150, 1]),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_and_backward(dtype, case):
    say(f"attention {dtype} {case}")
    Problem(dtype, seed=11, **case).check()


# rows enough for the larger tiles (128 rows of a workgroup, 256 in the last two; fp32: 64) on a device of up to 256 compute units
@pytest.mark.parametrize("case", [
    dict(heads=16, kv=16, d=64, ql=[129, 257, 1, 190] * 9, borders=LOG),
    dict(heads=16, kv=16, d=128, ql=[200, 77, 130, 65] * 9, causal=True),
    dict(heads=32, kv=16, d=32, ql=[200, 77, 130, 65] * 9, causal=True, borders=LOG),
    dict(heads=16, kv=16, d=128, ql=[200, 77, 130, 65] * 9, borders=[1, 4, 60]),
    dict(heads=16, kv=4, d=64, ql=[129, 257, 1, 190] * 9, causal=True),
    dict(dtype="f32", heads=16, kv=8, d=64, ql=[129, 257, 1, 190] * 5, borders=LOG),
    dict(dtype="f32", heads=16, kv=16, d=128, ql=[129, 257, 1, 190] * 5, causal=True),
    dict(heads=32, kv=8, d=64, ql=[1100, 1030], borders=[1, 2, 70, 300]),
    dict(heads=32, kv=32, d=128, ql=[1030, 1100]),
], ids=["64", "128c", "32c", "128b", "64c", "f32", "f32c", "256", "256w"])
def test_large_tiles(case):
    say(f"attention, large tiles {case}")
    Problem(**{"dtype": "bf16", "seed": 12, **case}).check()


@pytest.mark.parametrize("case", [dict(dtype="f32", heads=2, kv=2, ql=[300, 1200]), dict(dtype="bf16", heads=2, kv=1, ql=[300, 1200]),
                                  dict(dtype="bf16", heads=32, kv=32, ql=[1100, 1100])], ids=["f32", "bf16", "bf16 many"])
@pytest.mark.parametrize("causal", [False, True])
def test_borders_as_far_as_they_go(case, causal):
    """The bias gradient's sums by distance at their longest, heads of 128: they leave room for fewer wavefronts."""
    say(f"far borders {case} {causal}")
    Problem(d=128, causal=causal, borders=[1, 2, 500, 1023, 1024], seed=43, **case).check()


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("n", [100, 150, 1100])
def test_more_sequences_than_lanes(few, n):
    """Sequences by the hundred, some empty: a wavefront looks its own up 64 at a time, or in a table made for the call."""
    gen = torch.Generator().manual_seed(40)
    most = (2600 if n < 1000 else 40) if few else 60 if n < 1000 else 12
    kl = [int(x) for x in torch.randint(0, most, (n,), generator=gen)]
    ql = [int(x) for x in torch.randint(0, 3, (n,), generator=gen)] if few else [x + int(y) for x, y in zip(kl, torch.randint(0, 40, (n,), generator=gen))]
    Problem("bf16", 4 if few else 8, 2, 32, ql, kl, causal=True, borders=[1, 5, 30], seed=41, train=not few or n > 1000).check()


@pytest.mark.parametrize("case", [dict(heads=4, kv=2, d=64, ql=[150, 70]), dict(heads=8, kv=2, d=64, ql=[1, 1], kl=[4000, 1000])], ids=["tiles", "few"])
def test_a_stream_of_its_own(case):
    """stream=: work, workspaces and results are that stream's, whatever the current one is busy with."""
    p = Problem("bf16", causal=True, seed=42, tail=0, **case)
    want = p.run()
    q, k, v, dout, kw, qs, ks = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda(), p.kw(), dev(p.qs), dev(p.ks)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn((2048, 2048), device="cuda")
    got = []
    for _ in range(6):
        busy = (busy @ busy).clamp(-1, 1)                          # allocates and frees on the current stream
        out, lse = dchag.dchag_attend(q, k, v, qs, ks, stream=side, **kw)
        got.append([out, lse, *dchag.dchag_attend_backward(q, k, v, out, lse, dout, qs, ks, stream=side, **kw)[:3]])
    torch.cuda.synchronize()
    for g in got:
        for name, t in zip(("out", "lse", "dq", "dk", "dv"), g):
            assert torch.equal(t, want[name]), name


FEW = [
    dict(heads=8, kv=8, d=32, ql=[1] * 4, kl=[512] * 4, used=[128, 77, 300, 1], causal=True),
    dict(heads=8, kv=2, d=128, ql=[1] * 3, kl=[5000, 3, 2049], causal=True, borders=LOG),
    dict(heads=4, kv=1, d=64, ql=[5, 0, 3, 1], kl=[900, 40, 2, 0], causal=True, borders=[1, 2, 700]),
    dict(heads=16, kv=1, d=24, ql=[2, 1], kl=[700, 1500]),
    dict(heads=2, kv=2, d=64, ql=[7, 20], kl=[1111, 33], borders=LOG),
    dict(heads=32, kv=1, d=128, ql=[1], kl=[9000], causal=True, used=[8999]),
]


@pytest.mark.parametrize("case", FEW, ids=[str(i) for i in range(len(FEW))])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens_against_a_cache(dtype, case):
    say(f"attention of few rows {dtype} {case}")
    Problem(dtype, seed=13, **case).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("few", [False, True])
def test_values_at_masked_places_have_no_part(dtype, few):
    """A later token that is not finite: rows before it are as if it were not there, rows from it on are not finite."""
    p = Problem(dtype, 2, 1, 64, [200] if not few else [6], [200], causal=True, seed=14)
    at = 130 if not few else 196
    p.v[at], p.v[at + 1, 0, 3] = float("nan"), float("inf")
    p.dout = None
    want = p.want()
    assert torch.isfinite(want["out"][0][p.in_q][: at - 200]).all() if not few else True
    p.check(want=want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_at_masked_places_have_no_part(dtype):
    """A row of dout that is not finite reaches the keys that its query sees and no others."""
    p = Problem(dtype, 2, 1, 32, [200], causal=True, seed=15)
    p.dout[70] = float("nan")
    got = p.run()
    clean = Problem(dtype, 2, 1, 32, [200], causal=True, seed=15)
    want = clean.want()
    for name in ("dk", "dv"):
        g = got[name][:200].cpu()
        assert bool(g[:71].isnan().all()), name
        ref.check(name, g[71:], *(x[71:200] for x in want[name]))
    assert bool(got["dq"][70].isnan().all())
    rest = torch.arange(200) != 70
    ref.check("dq", got["dq"][:200].cpu()[rest], *(x[:200][rest] for x in want["dq"]))


@pytest.mark.parametrize("value", [float("-inf"), torch.finfo(torch.bfloat16).min])
@pytest.mark.parametrize("causal", [False, True])
def test_bias_that_masks(value, causal):
    """Buckets masked by -inf or by the type's lowest value; with all near ones masked, the first rows see nothing."""
    p = Problem("bf16", 2, 2, 64, [90, 20], causal=causal, borders=[1, 2, 30], seed=16)
    p.bias[0, :3] = value
    p.bias[1, 1] = value
    if not causal:
        p.bias[0, 4:] = value
    p.check()


def test_columns_of_one_tensor():
    """q, k and v are columns of one tensor, and so are their gradients; out and dout have rows with gaps."""
    h, hk, d, lens = 4, 2, 64, [130, 67]
    p = Problem("bf16", h, hk, d, lens, causal=True, borders=LOG, seed=17, tail=0)
    t, w = sum(lens), (h + 2 * hk) * d
    qkv, dqkv = torch.cat([x.flatten(1) for x in (p.q, p.k, p.v)], 1).cuda(), torch.full((t, w + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    cut = lambda x: (x[:, :h * d].view(t, h, d), x[:, h * d:(h + hk) * d].view(t, hk, d), x[:, (h + hk) * d:w].view(t, hk, d))  # noqa: E731
    wide_out, wide_dout = torch.full((t, h * d + 16), 7.0, dtype=torch.bfloat16, device="cuda"), torch.zeros((t, h * d + 8), dtype=torch.bfloat16, device="cuda")
    out, dout = wide_out[:, :h * d].view(t, h, d), wide_dout[:, 8:].view(t, h, d)
    dout.copy_(p.dout)
    q, k, v = cut(qkv)
    dq, dk, dv = cut(dqkv)
    out, lse = dchag.dchag_attend(q, k, v, dev(p.qs), dev(p.ks), out=out, **p.kw())
    _, _, _, db = dchag.dchag_attend_backward(q, k, v, out, lse, dout, dev(p.qs), dev(p.ks), dq=dq, dk=dk, dv=dv, **p.kw())
    p.check(got={"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dbias": db})
    assert bool((wide_out[:, h * d:] == 7).all()) and bool((dqkv[:, w:] == 7).all())


def test_cache_past_32_bits():
    """Key rows whose offsets pass 2^31 elements (rows 2^22 elements apart), for the split kernel and for the tiled one."""
    ld, rows, hk, d = 1 << 22, 620, 1, 64
    room = torch.zeros((rows * ld,), dtype=torch.bfloat16, device="cuda")
    k, v = room.view(rows, ld)[:, :d].unsqueeze(1), room.view(rows, ld)[:, d:2 * d].unsqueeze(1)
    gen = torch.Generator().manual_seed(18)
    kh, vh = normal(gen, "bf16", rows, hk, d), normal(gen, "bf16", rows, hk, d)
    k.copy_(kh), v.copy_(vh)
    for ql, kl in (([1, 1], [20, 600]), ([100], [620])):
        q = normal(gen, "bf16", sum(ql), 2, d)
        want = ref.attention(q, kh, vh, starts(ql), starts(kl), causal=True)
        out, lse = dchag.dchag_attend(q.cuda(), k, v, dev(starts(ql)), dev(starts(kl)), causal=True)
        ref.check("out", out, *want["out"])
        ref.check("lse", lse, *want["lse"])


def test_starts_beyond_the_tensors_stay_inside():
    """Starts and used counts outside the tensors are taken as the nearest inside."""
    p = Problem("bf16", 2, 1, 64, [60, 80], causal=True, seed=19, tail=0)
    q, k, v = p.q.cuda(), p.k.cuda(), p.v.cuda()
    want = dchag.dchag_attend(q, k, v, dev([0, 60, 140]), dev([0, 60, 140]), causal=True)
    got = dchag.dchag_attend(q, k, v, dev([-5, 60, 10 ** 9]), dev([-(2 ** 31), 60, 2 ** 31 - 1]), causal=True, k_used=dev([10 ** 9, 10 ** 9]))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_nothing_to_do():
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    bias = torch.ones((2, 2), dtype=torch.bfloat16, device="cuda")
    out, lse = dchag.dchag_attend(e(0, 2, 64), e(0, 1, 64), e(0, 1, 64), dev([0, 0]), dev([0, 0]))
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    kw = dict(causal=True, bias=bias, borders=[4])
    got = dchag.dchag_attend_backward(e(0, 2, 64), e(0, 1, 64), e(0, 1, 64), out, lse, e(0, 2, 64), dev([0, 0]), dev([0, 0]), **kw)
    assert bool((got[3] == 0).all())
    q = torch.ones((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = dchag.dchag_attend(q, e(0, 1, 64), e(0, 1, 64), dev([0, 5]), dev([0, 0]))
    assert bool((out == 0).all()) and bool((lse == float("-inf")).all())
    dq, _, _, _ = dchag.dchag_attend_backward(q, e(0, 1, 64), e(0, 1, 64), out, lse, q, dev([0, 5]), dev([0, 0]))
    assert bool((dq == 0).all())


SAME = [dict(heads=4, kv=2, d=64, ql=[150, 70], causal=True, borders=LOG), dict(heads=8, kv=2, d=128, ql=[1, 1], kl=[4000, 1000], borders=LOG)]


@pytest.mark.parametrize("case", SAME, ids=["tiles", "few"])
def test_same_bits_every_time_and_on_another_stream(case):
    p = Problem("bf16", seed=20, **case)
    one = p.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = p.run()
    side.synchronize()
    for n in one:
        assert torch.equal(one[n], two[n]) or bool((one[n].isnan() == two[n].isnan()).all()), n


@pytest.mark.parametrize("case", SAME, ids=["tiles", "few"])
def test_captured_and_replayed(case):
    """A training step in a graph, replayed on new inputs with eager work between, against the eager calls bit for bit."""
    p = Problem("bf16", seed=21, tail=0, **case)
    q, k, v, dout, kw = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.dout.cuda(), p.kw()
    qs, ks = dev(p.qs), dev(p.ks)

    def step():
        out, lse = dchag.dchag_attend(q, k, v, qs, ks, **kw)
        return [out, lse, *dchag.dchag_attend_backward(q, k, v, out, lse, dout, qs, ks, **kw)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        gen = torch.Generator().manual_seed(30 + i)
        for t in (q, k, v, dout):
            t.copy_(torch.randn(t.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_gradients_against_differences():
    """Directional derivatives of <dout, out> by central differences of the 64-bit form."""
    p = Problem("f32", 2, 1, 16, [23, 9], causal=True, borders=[1, 3, 7], seed=22, tail=0)
    got = p.run()
    gen = torch.Generator().manual_seed(23)

    def loss(q, k, v, bias):
        o = ref.attention(q, k, v, p.qs, p.ks, True, 0.0, None, bias, p.borders)["out"][0]
        return float((o * p.dout.double()).sum())

    base = [p.q.double(), p.k.double(), p.v.double(), p.bias.double()]
    for i, name in enumerate(("dq", "dk", "dv", "dbias")):
        way = torch.randn(base[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + h * way, base[i] - h * way
        want = (loss(*up) - loss(*down)) / (2 * h)
        have = float((got[name].double().cpu() * way).sum())
        size = float((got[name].double().cpu().abs() * way.abs()).sum())
        assert abs(have - want) <= 1e-5 * size + 1e-6, (name, have, want)        # differences: h^2, and fp32 gradients


def test_bias_without_its_gradient():
    p = Problem("bf16", 2, 2, 64, [100, 300], borders=LOG, seed=25, tail=0)
    q, k, v, qs, ks = p.q.cuda(), p.k.cuda(), p.v.cuda(), dev(p.qs), dev(p.ks)
    out, lse = dchag.dchag_attend(q, k, v, qs, ks, **p.kw())
    dq, dk, dv, db = dchag.dchag_attend_backward(q, k, v, out, lse, p.dout.cuda(), qs, ks, want_dbias=False, **p.kw())
    assert db is None
    want = p.want()
    del want["dbias"]
    p.check(got={"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, want=want)


def test_scale_of_ones_own():
    Problem("bf16", 2, 2, 64, [100], scale=0.3, borders=LOG, seed=24).check()
