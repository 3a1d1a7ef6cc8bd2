"""Products of microscaled 4-bit matrices, against sums in 64 bits."""
import math

import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import mx as X

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# one row and few, tiles of 16, 64, 128 and 256 and their neighbours, one column, sums of one element and of parts of a step
SHAPES = [(1, 1, 1), (1, 5, 128), (1, 1000, 640), (2, 16, 33), (3, 17, 129), (5, 300, 2049), (16, 64, 1000), (17, 65, 256), (31, 33, 384), (33, 129, 127), (64, 64, 128),
          (65, 255, 300), (100, 1, 500), (128, 257, 512), (129, 128, 1100), (256, 256, 256), (257, 300, 130), (300, 513, 640), (520, 260, 90)]


def grid(rng, rows, cols):
    """Values that need no rounding under a scale of 1, whose sums of products are multiples of 0.25 below 36 cols: exact in 32 bits in any order."""
    x = R.GRID[rng.integers(0, 8, (rows, cols))] * rng.choice([-1.0, 1.0], (rows, cols))
    return torch.from_numpy(x)


def held(x):
    """A matrix of these values, whose buffers have bytes of their own (NaN scales among them) in the rows that fill up a tile."""
    rows, cols = x.shape
    codes = np.zeros((rows, (cols + 127) // 128 * 128), dtype=np.uint8)
    a = x.abs().numpy()
    codes[:, :cols] = np.searchsorted(R.GRID, a) | np.where(np.signbit(x.numpy()), 8, 0).astype(np.uint8)
    scales = np.full((rows, codes.shape[1] // 32), 127)
    c, s = R.buffers(codes, scales, rows, cols, fill=0xFF)
    return X.MxMatrix(rows, cols, c.to(DEV), s.to(DEV))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_exact_sums(shape, dtype):
    (m, n, k), kind, h = shape, DTYPES[dtype], X.Mx()
    rng = np.random.default_rng(m * 1000003 + n * 1009 + k)
    a, b = grid(rng, m, k), grid(rng, n, k)
    want = a @ b.t()
    bias = torch.from_numpy(rng.integers(-64, 64, n) / 4.0).float()
    A, Bm = held(a), held(b)
    for with_bias in (False, True):
        for accumulate in (False, True):
            wide = torch.full((m, n + 7), 3.0, dtype=kind, device=DEV)
            out = wide[:, 3:3 + n]
            h.mc_mx_matmul(A, Bm, out, bias=bias.to(DEV) if with_bias else None, accumulate=accumulate)
            exact = want + (bias.double() if with_bias else 0.0) + (3.0 if accumulate else 0.0)
            assert torch.equal(out.cpu(), exact.float().to(kind)), (with_bias, accumulate)
            assert bool((wide[:, :3] == 3).all() and (wide[:, 3 + n:] == 3).all())
    h.close()


@pytest.mark.parametrize("shape", [(5, 30, 40000), (40, 33, 50000), (70, 100, 20000), (130, 70, 9000), (2700, 2600, 300), (2817, 2561, 130), (200, 330, 12000), (129, 4099, 1000), (1000, 1030, 1100), (9, 13000, 700),
                                   (30, 12900, 300), (50, 13001, 260), (67, 12950, 100)], ids=str)
def test_large_and_long(shape):
    """Sums that several blocks share, and outputs of many blocks, in each of the forms."""
    (m, n, k), h = shape, X.Mx()
    rng = np.random.default_rng(m + n + k)
    a, b = grid(rng, m, k), grid(rng, n, k)
    want = (a @ b.t()).float()
    bias = torch.from_numpy(rng.integers(-64, 64, n) / 4.0).float()
    A, Bm = held(a), held(b)
    for kind in (torch.float32, torch.bfloat16):
        out = torch.empty(m, n, dtype=kind, device=DEV)
        h.mc_mx_matmul(A, Bm, out)
        assert torch.equal(out.cpu(), want.to(kind))
        h.mc_mx_matmul(A, Bm, out, bias=bias.to(DEV), accumulate=True)
        assert torch.equal(out.cpu(), (want.to(kind).double() + want.double() + bias.double()).float().to(kind))


def test_very_long_sums():
    """More steps than the forms through LDS take."""
    h, (m, n, k) = X.Mx(), (66, 3, 2 ** 23 + 133)
    a, b = torch.zeros(m, k, dtype=torch.bfloat16, device=DEV), torch.zeros(n, k, dtype=torch.bfloat16, device=DEV)
    at = [0, 2 ** 23 - 1, 2 ** 23, k - 1]
    for i, c in enumerate(at):
        a[:, c], b[:, c] = float(2 ** i), 1.0
    a[65], b[2] = 2 * a[0], 4 * b[0]
    A, Bm, out = X.MxMatrix(m, k), X.MxMatrix(n, k), torch.empty(m, n, device=DEV)
    h.mc_mx_quantize(a, by_rows=A)
    h.mc_mx_quantize(b, by_rows=Bm)
    h.mc_mx_matmul(A, Bm, out)
    want = torch.full((m, n), 15.0)
    want[65] *= 2
    want[:, 2] *= 4
    assert torch.equal(out.cpu(), want)
    del a, b, A, Bm
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shape", [(1, 70, 5000), (40, 70, 2900), (130, 260, 1500), (300, 260, 9000), (3000, 2600, 600)], ids=str)
def test_rounded_sums(shape):
    """Scales over a wide range.  Each of the steps' sums of 128 products and the additions that join them is off by at most a few units of its terms' size: a
    matrix instruction adds 128 products in at least seven levels and its result to a sum, so 8 roundings of up to 2^-23 each."""
    (m, n, k), h = shape, X.Mx()
    rng = np.random.default_rng(7)
    a, b = (torch.from_numpy(rng.standard_normal((r, k)) * np.exp2(rng.integers(-12, 12, (r, k)))) for r in (m, n))
    mats = []
    for x in (a, b):
        codes, scales = R.quantized(x)
        c, s = R.buffers(codes, scales, *x.shape)
        mats.append(X.MxMatrix(*x.shape, c.to(DEV), s.to(DEV)))
    x, y = (R.matrix(q) for q in mats)
    out = torch.empty(m, n, device=DEV)
    h.mc_mx_matmul(*mats, out)
    off = (x.abs() @ y.abs().t()) * 8 * ((k + 127) // 128 + 64) * 2.0 ** -23 / 4
    assert bool(((out.cpu().double() - x @ y.t()).abs() <= off).all())


def test_blocks_that_stand_for_nan():
    """A NaN of a reaches its row, one of b its column, and nothing else."""
    for m, n, k in ((3, 40, 300), (70, 300, 300), (300, 280, 200), (600, 700, 1400), (2900, 2800, 600)):
        h, rng = X.Mx(), np.random.default_rng(9)
        a, b = grid(rng, m, k), grid(rng, n, k)
        x, y = a.to(DEV).float(), b.to(DEV).float()
        x[2, 100], y[n - 1, k - 1] = math.nan, math.inf
        A, Bm = X.MxMatrix(m, k), X.MxMatrix(n, k)
        h.mc_mx_quantize(x, by_rows=A)
        h.mc_mx_quantize(y, by_rows=Bm)
        out = torch.zeros(m, n, device=DEV)
        h.mc_mx_matmul(A, Bm, out)
        want = torch.zeros(m, n, dtype=torch.bool)
        want[2], want[:, n - 1] = True, True
        assert torch.equal(torch.isnan(out).cpu(), want)


def test_scales_at_the_ends():
    """Products of scales beyond and below 32 bits' range."""
    h = X.Mx()
    one = np.full((1, 128), 2, dtype=np.uint8)                      # ones
    for sa, sb, want in ((0, 254, 128.0), (254, 0, 128.0), (0, 0, 0.0), (254, 254, math.inf), (127, 127, 128.0), (254, 127, math.inf), (0, 127, 128.0 * 2.0 ** -127)):
        A, Bm = (X.MxMatrix(1, 128, *(t.to(DEV) for t in R.buffers(one, np.full((1, 4), s), 1, 128))) for s in (sa, sb))
        out = torch.empty(1, 1, device=DEV)
        h.mc_mx_matmul(A, Bm, out)
        assert float(out) == want, (sa, sb)


def test_nothing_to_do():
    h = X.Mx()
    h.mc_mx_matmul(X.MxMatrix(0, 100), X.MxMatrix(30, 100), torch.empty(0, 30, device=DEV))
    h.mc_mx_matmul(X.MxMatrix(30, 100), X.MxMatrix(0, 100), torch.empty(30, 0, device=DEV))


def test_same_bits_every_time():
    h, rng = X.Mx(), np.random.default_rng(3)
    for m, n, k in ((1, 200, 20000), (30, 100, 9000), (200, 300, 5000), (300, 330, 12000)):
        x = torch.from_numpy(rng.standard_normal((m, k))).float().to(DEV)
        y = torch.from_numpy(rng.standard_normal((n, k))).float().to(DEV)
        A, Bm = X.MxMatrix(m, k), X.MxMatrix(n, k)
        h.mc_mx_quantize(x, by_rows=A)
        h.mc_mx_quantize(y, by_rows=Bm)
        outs = [torch.empty(m, n, device=DEV) for _ in range(10)]
        for out in outs:
            h.mc_mx_matmul(A, Bm, out)
        assert all(torch.equal(outs[0], o) for o in outs)


def test_on_a_stream_and_in_a_graph():
    """Captured products of several forms, replayed between eager ones on the same handle."""
    h, rng = X.Mx(), np.random.default_rng(4)
    shapes = [(1, 300, 5000), (20, 70, 9000), (140, 300, 700), (200, 330, 12000)]
    mats = [(held(grid(rng, m, k)), held(grid(rng, n, k))) for m, n, k in shapes]
    outs = [torch.zeros(m, n, device=DEV) for m, n, _ in shapes]
    want = [torch.empty_like(o) for o in outs]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for (a, b), o in zip(mats, outs):
            h.mc_mx_matmul(a, b, o, accumulate=True)
    for (a, b), w in zip(mats, want):
        h.mc_mx_matmul(a, b, w)
    for i in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, i * w) for o, w in zip(outs, want)), i
        eager = [torch.empty_like(o) for o in outs]
        for (a, b), o in zip(mats, eager):
            h.mc_mx_matmul(a, b, o, stream=side)
        side.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(eager, want))


def test_outputs_beyond_31_bits():
    """Rows and elements of the result whose places pass 32 bits."""
    h, rng = X.Mx(), np.random.default_rng(5)
    m, n, k = 70000, 40000, 32
    a, b = grid(rng, m, k), grid(rng, n, k)
    out = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    h.mc_mx_matmul(held(a), held(b), out)
    for r in (0, 1, 53687, 53688, m - 1):
        assert torch.equal(out[r].cpu(), (a[r] @ b.t()).float().bfloat16()), r
    del out
    torch.cuda.empty_cache()


def test_refusals():
    h = X.Mx()
    a, b, out = X.MxMatrix(20, 100), X.MxMatrix(30, 100), torch.empty(20, 30, device=DEV)
    for bad in ((a, X.MxMatrix(30, 101), out), (a, b, out[:, :29]), (a, b, out[:19]), (a, b, out.t()), (a, b, out.double()), (a, b, out.cpu()), (a, b.codes, out), (b, a, out)):
        with pytest.raises(ValueError):
            h.mc_mx_matmul(*bad)
    for bias in (torch.empty(29, device=DEV), torch.empty(30), torch.empty(30, device=DEV, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            h.mc_mx_matmul(a, b, out, bias=bias)
    with pytest.raises(B.McError) as e:                       # the result over an operand
        h.mc_mx_matmul(a, X.MxMatrix(16, 100), a.codes.view(torch.float32)[:20 * 16].view(20, 16))
    assert e.value.status == B.MC_ERR_INVALID_ARG
    with pytest.raises(B.McError):
        h.mc_mx_matmul(a, b, out, bias=out[0])
