"""Plain 64-bit statements of the operators in mergecomp_mx.h, on the CPU (not collected by pytest), from the header's definitions alone."""
import math

import numpy as np
import torch

F64 = torch.float64
LOST = 2.0 ** -63                 # the root of a second moment that may count as 0, 2^-126
U = 2.0 ** -24                    # half a unit in the last place of binary32, relative
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
UP_AT = np.array([False, True, False, True, False, True, False])        # a border itself goes to the neighbour with the even code


# ---- moments in 8 bits
def value8(code):
    """An 8-bit float, from its fields."""
    c = code.cpu().numpy().astype(np.int64)
    e, m = c >> 3 & 15, (c & 7).astype(np.float64)
    x = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    x = np.where(c & 127 == 127, np.nan, x)
    return torch.from_numpy(np.where(c & 128, -x, x))


def spread(scale, n):
    """A block's scale for each of its elements."""
    return scale.cpu().to(F64).repeat_interleave(128)[:n]


def half_step8(y):
    """What rounding y to an 8-bit float may change."""
    y = y.abs().clamp(min=2.0 ** -6)
    return torch.exp2(torch.floor(torch.log2(y)) - 4)


def adamw8(p, cm, sm, cr, sr, g, coef, step, lr, betas, eps, decay):
    """(p, m, r) after the update, before the moments are rounded, and what 32-bit arithmetic may be off by in each."""
    n = p.numel()
    p, g = p.cpu().to(F64), g.cpu().to(F64) * coef
    m, r = value8(cm) * spread(sm, n), value8(cr) * spread(sr, n)
    b1, b2 = betas
    m_new = b1 * m + (1 - b1) * g
    v_new = b2 * r * r + (1 - b2) * g * g
    root = torch.sqrt(v_new)
    den = root / math.sqrt(1 - b2 ** step) + eps
    rate = lr / (1 - b1 ** step)
    p_new = p - lr * decay * p - rate * m_new / den
    # m: a held value is off by U, g by U, each product by two more with its constant, the sum by one; its terms may cancel.  v: squares of
    # what is off by U by 3 U, with their factors 5 U, the sum 6 U; the root half of that and 2 U of its own (a unit in the last place).  p: the quotient has m's
    # error, the root's, and 6 U of product, sum, quotient and rate; its difference from p's product 4 U.
    size = (b1 * m).abs() + ((1 - b1) * g).abs()
    tiny = 2.0 ** -140
    off_m, off_r = 5 * U * size + tiny, 5 * U * root + LOST
    off_p = 4 * U * p.abs() + rate * (20 * U * size + tiny) / den + rate * m_new.abs() / den ** 2 * LOST
    return (p_new, m_new, root), (off_p, off_m, off_r)


def check8(x, off, code, scale, root):
    """Whether codes and scales hold x, known up to `off`, as the header says; a text of what is wrong, or nothing."""
    n = x.numel()
    for b in range(0, n, 128):
        xs, os, s = x[b:b + 128], off[b:b + 128], float(scale[b // 128])
        fine = torch.isfinite(xs)
        c = value8(code[b:b + 128])
        if not torch.equal(torch.isnan(c), ~fine):
            return f"block {b // 128}: NaN elsewhere"
        xs, os, c = xs[fine], os[fine], c[fine]
        top = float(xs.abs().max()) if xs.numel() else 0.0
        if top < 2.0 ** -100 * (1 - 2.0 ** -20):
            if s != 0 or bool((c != 0).any()):
                return f"block {b // 128}: not zeros"
            continue
        if abs(s - top / 448) > (float(os.max()) + 3 * U * top) / 448:
            return f"block {b // 128}: scale {s}, largest {top}"
        y = xs / s
        least = torch.where((xs > 0) & (y < 2.0 ** -9), 2.0 ** -9 - y, 0.0) if root else 0.0
        bad = (c - y).abs() > torch.maximum(half_step8(y), torch.as_tensor(least, dtype=F64)) * (1 + 2.0 ** -20) + os / s + 4 * U * y.abs()
        if root:
            bad |= (xs > os) & (c == 0)
        if bool(bad.any()):
            i = int(torch.nonzero(bad)[0])
            return f"block {b // 128}: {float(y[i])} held as {float(c[i])}"
    return ""


# ---- microscaled matrices
def places(rows, cols):
    """Where, by the header's formulas, the code of every element lies (byte, and whether in its high half), and the scale of every block."""
    steps = (cols + 127) // 128
    r, c = np.arange(rows, dtype=np.int64)[:, None], np.arange(steps * 128, dtype=np.int64)[None, :]
    s, g, i = c // 128, c % 128 // 32, c % 32
    byte = (((r // 16) * steps + s) * 64 + g * 16 + r % 16) * 16 + i // 2
    k = np.arange(steps * 4, dtype=np.int64)[None, :]
    scale = (((r // 64) * steps + k // 4) * 64 + k % 4 * 16 + r % 16) * 4 + r // 16 % 4
    return byte, i % 2 + 0 * r, scale


def taken_apart(m):
    """(codes rows x padded columns, scales rows x blocks) of an MxMatrix."""
    byte, high, scale = places(m.rows, m.cols)
    codes, scales = m.codes.cpu().numpy(), m.scales.cpu().numpy()
    return codes[byte] >> (4 * high).astype(np.uint8) & 15, scales[scale].astype(np.int64)


def values4(codes, scales):
    x = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.repeat(np.where(scales == 255, np.nan, np.exp2(scales - 127.0)), 32, 1)
    return torch.from_numpy(x)


def matrix(m):
    """An MxMatrix's values, without its padding."""
    return values4(*taken_apart(m))[:, :m.cols]


def quantized(x):
    """(codes, scales) of a matrix whose rows are padded to 128 columns, in exact arithmetic."""
    x = x.detach().cpu().to(F64).numpy()
    rows, cols = x.shape
    full = np.zeros((rows, (cols + 127) // 128 * 128))
    full[:, :cols] = x
    blocks = full.reshape(rows, -1, 32)
    top = np.abs(blocks).max(2)
    odd = ~np.isfinite(top)
    m, e = np.frexp(np.where(odd, 0.0, top))                             # m in [0.5, 1), so that fraction = 2 m and E = e - 1
    scale = np.where(top == 0, -127, np.maximum(e - 1 - np.where(2 * m <= 1.75, 2, 1), -127))
    y = np.abs(np.where(odd[:, :, None], 0.0, blocks)) / np.exp2(scale.astype(np.float64))[:, :, None]
    code = np.zeros(y.shape, dtype=np.uint8)
    for border, up in zip(BORDERS, UP_AT):
        code += (y >= border) if up else (y > border)
    code |= np.where(np.signbit(blocks) & ~odd[:, :, None], 8, 0).astype(np.uint8)
    return code.reshape(rows, -1), np.where(odd, 255, scale + 127)


def rounded(x, kind):
    """Values in the type, those beyond its range as its largest."""
    most = torch.finfo(kind).max
    return torch.where(torch.isnan(x), x, x.clamp(-most, most)).to(kind)


def packed(values, cols=None):
    """Buffers of a matrix whose values are of the grid itself (scales 1), rows x cols."""
    rows, cols = values.shape
    codes, scales = quantized(values)
    return buffers(codes, scales, rows, cols)


def buffers(codes, scales, rows, cols, fill=0xA5):
    """Codes and scales laid out; `fill` where nothing belongs (rows that fill up a tile)."""
    steps = (cols + 127) // 128
    byte, high, at = places(rows, cols)
    c = np.full((rows + 15) // 16 * steps * 1024, fill, dtype=np.uint8)
    s = np.full((rows + 63) // 64 * steps * 256, fill, dtype=np.uint8)
    c[byte[:, 0::2]] = codes[:, 0::2] | codes[:, 1::2] << 4
    s[at] = scales
    return torch.from_numpy(c), torch.from_numpy(s)
