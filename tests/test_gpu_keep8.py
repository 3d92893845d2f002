"""Rows kept in 8 bits: codes, exponents and values bit for bit against the format's 64-bit definition, and the weight gradient that reads
them within derived bounds."""
import pytest
import torch

import paper_2506_21411_amd as dchag

from . import spatial_reference as ref

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of(dtype, rows, D, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, D), generator=gen) * torch.exp(2 * torch.randn((rows, 1), generator=gen)) * torch.exp(torch.randn((1, D), generator=gen))
    return x.to(TDT[dtype])


def awkward(dtype):
    """Rows on borders: ties, the largest code, all zeros, one value, smallest and largest numbers of the type, values that are not finite."""
    x = torch.zeros((16, 40), dtype=torch.float64)
    x[0, :8] = torch.tensor([448.0, -448.0, 1.0625, 1.1875, -1.0625, 17.0, 19.0, 0.0625])
    x[1, 0] = 448.5
    x[2, 5] = -3.0
    x[3] = torch.linspace(-2, 2, 40)
    x[4, :6] = torch.tensor([2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 448.0, -2.0 ** -6, 7.5 * 2.0 ** -9])
    info = torch.finfo(TDT[dtype])
    x[5, :3] = torch.tensor([info.max, -info.max, 1.0])
    x[6, :3] = torch.tensor([info.tiny, -info.tiny / 2, info.tiny * 4])
    x[7, :4] = torch.tensor([float("inf"), 1.0, float("-inf"), float("nan")])
    x[8, 33] = float("nan")
    x[9] = 1e-30
    x[10] = 2.0 ** torch.arange(-20, 20, dtype=torch.float64)
    x[11] = -x[10] * 1.75
    x[12] = x[10] * 1.8125
    x[13, :2] = torch.tensor([1e38, 1e-38])
    return x.to(TDT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["awkward", (1, 8), (3, 24), (130, 96), (65, 1000), (257, 1024)])
def test_codes_and_values(dtype, shape):
    x = awkward(dtype) if shape == "awkward" else rows_of(dtype, *shape, seed=1)
    values, codes, held = ref.pack8(x)
    c, s = dchag.dchag_pack8(x.cuda())
    nan = ~torch.isfinite(x)
    assert torch.equal(s.cpu(), held)
    same = torch.equal(c.cpu()[~nan], codes[~nan]) and bool(((c.cpu()[nan] & 127) == 127).all())
    assert same
    back = dchag.dchag_unpack8(c, s, x.dtype).cpu()
    same = bool(back[nan].isnan().all()) and torch.equal(back[~nan], values[~nan].to(x.dtype))
    assert same
    off = (back[~nan].double() - x[~nan].double()).abs()
    small = (2.0 ** (held.double() - 137)).repeat_interleave(32, 1)[:, :x.shape[1]][~nan]
    # half a step of 3 mantissa bits, or of the smallest codes; the types' own smallest numbers round once more
    near = bool((off <= torch.maximum(x[~nan].double().abs() / 16, small) + torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps / 2).all())
    assert near


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_with_gaps(dtype):
    x = rows_of(dtype, 33, 136, 2)
    room = torch.full((33, 160), float("nan"), dtype=x.dtype, device="cuda")
    room[:, 8:144] = x.cuda()
    c, s = dchag.dchag_pack8(room[:, 8:144])
    c2, s2 = dchag.dchag_pack8(x.cuda())
    assert torch.equal(c, c2) and torch.equal(s, s2)
    to = torch.full((33, 144), 7.0, dtype=x.dtype, device="cuda")
    dchag.dchag_unpack8(c, s, out=to[:, :136])
    assert torch.equal(to[:, :136], dchag.dchag_unpack8(c, s, x.dtype)) and bool((to[:, 136:] == 7).all())


def weight_grad(dtype, rows, d_in, d_out, seed=3):
    gen = torch.Generator().manual_seed(seed)
    values, codes, held = ref.pack8(rows_of(dtype, rows, d_in, seed))
    dy = torch.randn((rows, d_out), generator=gen).to(TDT[dtype])
    u = ref.unit(dy.dtype)
    x, g = values.to(dy.dtype).double(), dy.double()
    dW, db = g.T @ x, g.sum(0)
    n = rows * ref.F32
    return dy, codes, held, (dW, n * (g.abs().T @ x.abs()) + u * dW.abs()), (db, n * g.abs().sum(0) + u * db.abs())


# the last sizes take squares of 128 and of 256 of dW on a device of up to 256 compute units
SIZES = [(1, 8, 8), (5, 40, 24), (64, 128, 128), (300, 136, 264), (1000, 1000, 72), (2100, 264, 136), (0, 16, 24), (6000, 392, 1000), (9000, 1032, 648)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_weight_gradient(dtype, size):
    dy, codes, held, dW, db = weight_grad(dtype, *size)
    got = dchag.dchag_weight_grad8(dy.cuda(), codes.cuda(), held.cuda())
    ref.check("dW", got[0], *dW)
    ref.check("db", got[1], *db)
    again = dchag.dchag_weight_grad8(dy.cuda(), codes.cuda(), held.cuda(), want_db=False)
    assert again[1] is None and torch.equal(again[0], got[0])


def test_weight_gradient_of_a_part_of_the_columns():
    dy, codes, held, dW, db = weight_grad("bf16", 500, 128, 64)
    room = torch.full((500, 96), float("nan"), dtype=dy.dtype, device="cuda")
    room[:, 16:80] = dy.cuda()
    got = dchag.dchag_weight_grad8(room[:, 16:80], codes.cuda(), held.cuda())
    ref.check("dW", got[0], *dW)
    ref.check("db", got[1], *db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradient_reads_every_code(dtype):
    """One row of dy picks one row of x: all codes at many exponents, the smallest and the largest among them, come out as they stand."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(64, 1)
    codes[codes & 127 == 127] = 0                                  # NaN
    held = torch.randint(30, 220, (64, 8), generator=torch.Generator().manual_seed(7)).to(torch.uint8)
    held[0], held[1], held[2] = 0, 1, 246
    want = dchag.dchag_unpack8(codes.cuda(), held.cuda(), torch.float32).cpu()
    byte = held.long().repeat_interleave(32, 1).double()
    c = codes.long()
    mag = torch.where(c & 127 < 8, (c & 7) / 8.0 * 2.0 ** -6, (1 + (c & 7) / 8.0) * torch.exp2(((c >> 3) & 15).double() - 7))
    value = torch.where(c > 127, -mag, mag) * torch.exp2(byte - 127)
    assert torch.equal(want.double(), value)
    dW, db = dchag.dchag_weight_grad8(torch.eye(64).to(TDT[dtype]).cuda(), codes.cuda(), held.cuda())
    tiny = torch.finfo(torch.float32).smallest_normal               # products below the normal numbers may come out as zero
    ok = (dW.double().cpu() == value.to(TDT[dtype]).double()) | (value.abs() < tiny)
    assert bool(ok.all()) and bool((db == 1).all())


def test_values_past_32_bits():
    """More than 2^31 values: the last rows come back as the first ones do."""
    D, rows = 2048, (1 << 20) + 5
    x = torch.zeros((rows, D), dtype=torch.bfloat16, device="cuda")
    some = rows_of("bf16", 5, D, 4).cuda()
    x[-5:] = some
    c, s = dchag.dchag_pack8(x)
    c5, s5 = dchag.dchag_pack8(some)
    assert torch.equal(c[-5:], c5) and torch.equal(s[-5:], s5)
    back = dchag.dchag_unpack8(c, s)
    assert torch.equal(back[-5:], dchag.dchag_unpack8(c5, s5)) and not bool(back[:-5].any())


def test_captured_and_replayed():
    x, dy = rows_of("bf16", 700, 256, 5).cuda(), rows_of("bf16", 700, 128, 6).cuda()

    def step():
        c, s = dchag.dchag_pack8(x)
        return [c, s, dchag.dchag_unpack8(c, s), *dchag.dchag_weight_grad8(dy, c, s)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(rows_of("bf16", 700, 256, 10 + i)), dy.copy_(rows_of("bf16", 700, 128, 20 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
