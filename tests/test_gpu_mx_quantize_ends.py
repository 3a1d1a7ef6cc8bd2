"""Microscaled 4-bit quantisation along the columns where places pass 31 bits, and the least numbers of the 16-bit types."""
import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import mx as X

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("shape,rows_too", [((19, 2 ** 28 + 33), False), ((19, 2 ** 28 + 33), True), ((2 ** 28 + 33, 5), False)], ids=str)
def test_places_beyond_31_bits(shape, rows_too):
    """Bytes of the transposed matrix's codes and, with the rows' blocks, of the second tile of 16 rows."""
    h, (rows, cols) = X.Mx(), shape
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    at = [(0, 0), (rows - 1, cols - 1), (rows - 1, 0), (rows // 2, cols // 2), (0, cols - 1)]
    for i, (r, c) in enumerate(at):
        x[r, c] = float(2 ** i) * 3.0

    def place(m, r, c):
        steps = (m.cols + 127) // 128
        byte = (((r // 16) * steps + c // 128) * 64 + c % 128 // 32 * 16 + r % 16) * 16 + c % 32 // 2
        return byte, (((r // 64) * steps + c // 128) * 64 + c % 128 // 32 * 16 + r % 16) * 4 + r // 16 % 4
    by_cols, by_rows = X.MxMatrix(cols, rows), (X.MxMatrix(rows, cols) if rows_too else None)
    values = torch.empty_like(x) if rows_too else None
    h.mc_mx_quantize(x, by_rows=by_rows, by_cols=by_cols, values=values)
    for m, where in ((by_cols, [(c, r) for r, c in at]), (by_rows, at)):
        if m is None:
            continue
        for i, (r, c) in enumerate(where):
            byte, scale = place(m, r, c)
            # 3 * 2^j, the largest of its block, is 6 times 2^(j - 1); 3 * 2^i there 6 / 2^(j - i) times it
            top = max(j for j, (p, q) in enumerate(where) if (p, q // 32) == (r, c // 32))
            code = {0: 7, 1: 5, 2: 3, 3: 2, 4: 1}[top - i]   # 6, 3, 1.5, 0.75 (half way, to the even code of 1), 0.375 (0.5)
            assert int(m.codes[byte]) >> (4 * (c % 2)) & 15 == code and int(m.scales[scale]) == 126 + top, (i, m.rows)
        assert int(torch.count_nonzero(m.codes)) == len({place(m, r, c)[0] for r, c in where})
    if values is not None:
        assert all(float(values[r, c]) == float(x[r, c]) for r, c in at) and int(torch.count_nonzero(values)) == len(at)
    h.close()
    del x, values, by_rows, by_cols
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16], ids=str)
def test_the_least_numbers(kind):
    """Blocks of numbers below the type's least normal one, and around it."""
    gen = torch.Generator()
    gen.manual_seed(4)
    bits = torch.randint(0, 1 << (8 if kind is torch.bfloat16 else 11), (70, 200), generator=gen)          # two exponents: 0, and the least normal one
    bits[20:40] %= 4                                         # the very least
    bits[:, 64:96] >>= 2
    sign = torch.randint(0, 2, (70, 200), generator=gen) << 15
    x = (bits | sign).to(torch.int32).to(torch.int16).view(kind).to(DEV)
    assert torch.equal(x.cpu().view(torch.int16).int() & 0xFFFF, (bits | sign).int())
    h, r, c, v = X.Mx(), X.MxMatrix(70, 200), X.MxMatrix(200, 70), torch.empty_like(x)
    h.mc_mx_quantize(x, by_rows=r, by_cols=c, values=v)
    for m, y in ((r, x), (c, x.t())):
        codes, scales = R.quantized(y)
        got_codes, got_scales = R.taken_apart(m)
        assert (got_scales == scales).all() and (got_codes == codes).all()
    assert torch.equal(v.cpu(), R.rounded(R.values4(*R.quantized(x))[:, :200], kind))
    only = X.MxMatrix(70, 200)
    h.mc_mx_quantize(x, by_rows=only)
    assert torch.equal(only.codes, r.codes) and torch.equal(only.scales, r.scales)
    h.close()
