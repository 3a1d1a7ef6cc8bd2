"""Products whose scales differ from block to block, in each of their forms."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import mx as X

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# up to 16, 32 and 64 rows against columns on both sides of where a block takes more of them (6400 and 12 800), sums that blocks share, small products of more
# rows, 128 x 128 and 256 x 256 outputs to a block
SHAPES = [(1, 1, 1), (3, 200, 700), (16, 6400, 129), (1, 6401, 300), (7, 9001, 2000), (16, 12799, 700), (16, 12800, 4096), (16, 12801, 300), (9, 13000, 7000), (5, 30, 7200),
          (17, 12800, 300), (30, 333, 900), (32, 12801, 260), (31, 33, 7200), (33, 12800, 200), (64, 12801, 300), (50, 13001, 260), (65, 70, 300), (67, 12950, 100), (61, 90, 7200),
          (65, 3000, 1500), (130, 70, 7200), (257, 513, 1300), (512, 1024, 3000), (2700, 2600, 300), (2817, 2561, 130)]


def held(rng, rows, cols, least, most):
    """A matrix of random codes under random scales from 2^least to 2^most, and its values; bytes of their own in the rows that fill up a tile."""
    codes = np.zeros((rows, (cols + 127) // 128 * 128), dtype=np.uint8)
    codes[:, :cols] = rng.integers(0, 16, (rows, cols))
    scales = rng.integers(127 + least, 128 + most, (rows, codes.shape[1] // 32))
    c, s = R.buffers(codes, scales, rows, cols, fill=0xFF)
    return X.MxMatrix(rows, cols, c.to(DEV), s.to(DEV)), R.values4(codes, scales)[:, :cols]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_exact_sums(shape):
    """Scales of 1/2, 1 and 2: products are multiples of 1/16 and at most 144, so that sums of up to 7281 of them are whole numbers of sixteenths below 2^24, exact in 32 bits in
    any order."""
    (m, n, k), h = shape, X.Mx()
    assert 144 * 16 * k < 2 ** 24
    rng = np.random.default_rng(m * 1000003 + n * 1009 + k)
    (a, x), (b, y) = held(rng, m, k, -1, 1), held(rng, n, k, -1, 1)
    want = (x @ y.t()).float()
    for kind in (torch.float32, torch.bfloat16):
        out = torch.empty(m, n, dtype=kind, device=DEV)
        h.mc_mx_matmul(a, b, out)
        assert torch.equal(out.cpu(), want.to(kind)), kind
    h.close()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rounded_sums(shape):
    """Scales over 24 powers of two.  A term goes through its step's matrix instruction (128 products in seven levels, and the sum before: 8 roundings of up to 2^-23, also
    where a step is two instructions of 64: 2 * (6 + 1) = 14), those of the steps behind it, and the joins: up to 8 wavefronts' or 2 groups' sums and up to 64
    parts, as many as steps.  Each rounding is of at most the terms' magnitudes added up."""
    (m, n, k), h = shape, X.Mx()
    rng = np.random.default_rng(m + n + k)
    (a, x), (b, y) = held(rng, m, k, -12, 12), held(rng, n, k, -12, 12)
    out = torch.empty(m, n, device=DEV)
    h.mc_mx_matmul(a, b, out)
    steps = (k + 127) // 128
    roundings = 14 * steps + 7 + min(steps, 64)
    off = (x.abs() @ y.abs().t()) * roundings * 2.0 ** -23
    assert bool(((out.cpu().double() - x @ y.t()).abs() <= off).all())
    h.close()
