"""Microscaled 4-bit quantisation, code by code against its definition."""
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
SHAPES = [(1, 1), (1, 128), (1, 129), (3, 31), (15, 32), (16, 33), (17, 127), (63, 96), (64, 128), (65, 257), (128, 128), (129, 300), (200, 64), (37, 1000)]


def values(rows, cols, kind, seed=1, gap=0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x = torch.randn(rows, cols + gap, device=DEV, generator=gen)
    x *= torch.exp2(torch.randint(-9, 3, (rows, cols + gap), device=DEV, generator=gen).float())
    # what lies on a border between two codes, or between two scales, and zeros
    some = torch.tensor([0.0, -0.0, 0.25, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -7.0, 7.03125, 6.0, 14.0, -0.5], device=DEV)
    pick = torch.randint(0, 4 * len(some), (rows, cols + gap), device=DEV, generator=gen)
    x = torch.where(pick < len(some), some[pick.clamp(max=len(some) - 1)], x)
    return x.to(kind)[:, :cols]


def matrix(rows, cols):
    """With bytes of its own where nothing is to be written."""
    m = X.MxMatrix(rows, cols)
    m.codes.fill_(0xA5)
    m.scales.fill_(0xA5)
    return m


def check(m, x):
    codes, scales = R.quantized(x)
    c, s = R.buffers(codes, scales, m.rows, m.cols)
    assert torch.equal(m.codes.cpu(), c)                     # (whole buffers: rows that fill up a tile are as they were)
    assert torch.equal(m.scales.cpu(), s)
    return R.values4(codes, scales)[:, :m.cols]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions(shape, dtype):
    (rows, cols), kind, h = shape, DTYPES[dtype], X.Mx()
    for gap in (0, 3):
        x = values(rows, cols, kind, gap=gap)
        for by in ("r", "c", "rc", "rv", "cv", "rcv", "v"):
            r, c = (matrix(rows, cols) if "r" in by else None), (matrix(cols, rows) if "c" in by else None)
            wide = torch.full((rows, cols + 5), 9.0, dtype=kind, device=DEV)
            v = wide[:, 2:2 + cols] if "v" in by else None
            h.mc_mx_quantize(x, by_rows=r, by_cols=c, values=v)
            if r is not None:
                check(r, x)
            if c is not None:
                check(c, x.t())
            if v is not None:
                assert torch.equal(v.cpu(), R.rounded(R.values4(*R.quantized(x))[:, :cols], kind)), by
                assert bool((wide[:, :2] == 9).all() and (wide[:, 2 + cols:] == 9).all())
    h.close()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_not_finite(dtype):
    """A block with an infinity or a NaN stands for NaN, its neighbours for themselves, in either direction."""
    kind, h = DTYPES[dtype], X.Mx()
    x = values(70, 200, kind)
    x[3, 5], x[64, 199], x[40, 64] = math.inf, math.nan, -math.inf
    r, c, v = matrix(70, 200), matrix(200, 70), torch.empty(70, 200, dtype=kind, device=DEV)
    h.mc_mx_quantize(x, by_rows=r, by_cols=c, values=v)
    want = check(r, x)
    check(c, x.t())
    assert int(torch.isnan(want).sum()) == 32 + 8 + 32
    torch.testing.assert_close(v.cpu(), R.rounded(want, kind), rtol=0, atol=0, equal_nan=True)


def test_ends_of_the_range():
    """The smallest and the largest numbers of 32 bits."""
    h = X.Mx()
    x = torch.zeros(8, 64, device=DEV)
    x[0, :3] = torch.tensor([2.0 ** -149, -2.0 ** -126, 2.0 ** -127], device=DEV)
    x[1, :2] = torch.tensor([2.0 ** -149, 2.0 ** -148], device=DEV)
    x[2, :4] = torch.tensor([torch.finfo(torch.float32).max, -1.75 * 2.0 ** 127, 2.0 ** 125, 2.0 ** 100], device=DEV)
    x[3, 32:35] = torch.tensor([2.0 ** -125 * 1.8, 2.0 ** -126 * 1.5, 2.0 ** -128], device=DEV)
    x[4, 31], x[4, 32] = 1.0, 2.0 ** -40
    r, v = matrix(8, 64), torch.empty(8, 64, device=DEV)
    h.mc_mx_quantize(x, by_rows=r, values=v)
    want = check(r, x)
    assert torch.equal(v.cpu(), R.rounded(want, torch.float32))
    y = torch.full((2, 40), 65504.0, dtype=torch.float16, device=DEV)
    y[1] = -61440.0
    r, v = matrix(2, 40), torch.empty_like(y)
    h.mc_mx_quantize(y, by_rows=r, values=v)
    want = check(r, y)
    assert bool((want[0] == 65536).all()) and bool((v[0] == 65504).all()) and torch.equal(v.cpu(), R.rounded(want, torch.float16))


@pytest.mark.parametrize("cols_too", [False, True])
def test_in_place(cols_too):
    h, x = X.Mx(), values(130, 170, torch.bfloat16, gap=6)
    was, r, c = x.clone(), matrix(130, 170), (matrix(170, 130) if cols_too else None)
    h.mc_mx_quantize(x, by_rows=r, by_cols=c, values=x)
    assert torch.equal(x.cpu(), R.rounded(check(r, was), torch.bfloat16))
    if cols_too:
        check(c, was.t())


def test_values_are_quantised_to_themselves():
    h, x = X.Mx(), values(100, 300, torch.float32)
    a, b, v, w = matrix(100, 300), matrix(100, 300), torch.empty(100, 300, device=DEV), torch.empty(100, 300, device=DEV)
    h.mc_mx_quantize(x, by_rows=a, values=v)
    h.mc_mx_quantize(v, by_rows=b, values=w)
    assert torch.equal(v, w) and torch.equal(R.matrix(a), R.matrix(b))


def test_no_rows():
    h = X.Mx()
    h.mc_mx_quantize(torch.empty(0, 50, device=DEV), by_rows=X.MxMatrix(0, 50), values=torch.empty(0, 50, device=DEV))


def test_long_rows_and_many_rows():
    """Places beyond 31 bits of a byte."""
    h = X.Mx()
    for rows, cols in ((3, 2 ** 29 + 33), (2 ** 25 + 3, 32)):
        x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
        at = [(0, 0), (rows - 1, cols - 1), (rows - 1, 0), (rows // 2, cols // 2)]
        for i, (r, c) in enumerate(at):
            x[r, c] = float(2 ** i) * 3.0
        m, v = X.MxMatrix(rows, cols), torch.empty_like(x)
        h.mc_mx_quantize(x, by_rows=m, values=v)
        assert torch.equal(x, v)
        steps = (cols + 127) // 128
        for i, (r, c) in enumerate(at):
            byte = (((r // 16) * steps + c // 128) * 64 + c % 128 // 32 * 16 + r % 16) * 16 + c % 32 // 2
            scale = (((r // 64) * steps + c // 128) * 64 + c % 128 // 32 * 16 + r % 16) * 4 + r // 16 % 4
            # 3 * 2^j, the largest of its block, is 6 times 2^(j - 1); half of it 3 times that (code 5)
            top = max(j for j, (p, q) in enumerate(at) if (p, q // 32) == (r, c // 32))
            assert int(m.codes[byte]) >> (4 * (c % 2)) & 15 == 7 - 2 * (top - i) and int(m.scales[scale]) == 126 + top, (rows, i)
        assert int(torch.count_nonzero(m.codes)) == len(at)
        del x, m, v
        torch.cuda.empty_cache()


def test_on_a_stream_and_in_a_graph():
    h, x = X.Mx(), values(300, 500, torch.bfloat16)
    a, b = [matrix(300, 500), matrix(500, 300)], [matrix(300, 500), matrix(500, 300)]
    h.mc_mx_quantize(x, *a)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h.mc_mx_quantize(x, *a)
    for i in range(3):
        x.mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        h.mc_mx_quantize(x, *b, stream=side)
        side.synchronize()
        assert all(torch.equal(p.codes, q.codes) and torch.equal(p.scales, q.scales) for p, q in zip(a, b)), i


def test_refusals():
    h, x = X.Mx(), values(20, 50, torch.float32)
    good = X.MxMatrix(20, 50)
    with pytest.raises(B.McError) as e:
        h.mc_mx_quantize(x)
    assert e.value.status == B.MC_ERR_INVALID_ARG
    for bad in (dict(by_rows=X.MxMatrix(50, 20)), dict(by_cols=good), dict(by_rows=X.MxMatrix(20, 49)), dict(by_rows=x), dict(by_rows=good, values=x[:, :49]),
                dict(by_rows=good, values=torch.empty(20, 50, device=DEV, dtype=torch.bfloat16)), dict(by_rows=good, values=torch.empty(20, 50))):
        with pytest.raises(ValueError):
            h.mc_mx_quantize(x, **bad)
    for bad in (x.t(), x[0], x.double(), x.cpu()):
        with pytest.raises(ValueError):
            h.mc_mx_quantize(bad, by_rows=good)
    wide = torch.empty(20, 60, device=DEV)
    with pytest.raises(B.McError):                            # results over what is read
        h.mc_mx_quantize(wide[:, :50], by_rows=good, values=wide[:, 1:51])
    with pytest.raises(B.McError):
        h.mc_mx_quantize(x, by_rows=good, by_cols=X.MxMatrix(50, 20, torch.zeros(4 * 1024, dtype=torch.uint8, device=DEV), good.scales))
    for wrong in (dict(codes=good.codes), dict(codes=good.codes[1:], scales=good.scales), dict(codes=good.codes.cpu(), scales=good.scales.cpu()),
                  dict(codes=good.codes, scales=good.scales.float())):
        with pytest.raises(ValueError):
            X.MxMatrix(20, 50, **wrong)
    for rows, cols in ((-1, 5), (5, 0), (2 ** 31, 5)):
        with pytest.raises(ValueError):
            X.MxMatrix(rows, cols)
