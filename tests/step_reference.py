"""Plain 64-bit statements of the operators in mergecomp_step.h, on the CPU (not collected by pytest).

They are written element by element from the definitions in the header, with no code of the package."""
import math

import torch

F64 = torch.float64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24                    # half a unit in the last place of binary32, relative


def norm(grads, scale, max_norm):
    total = sum(float((g.cpu().to(F64) ** 2).sum()) for g in grads)
    if not math.isfinite(total):
        return math.sqrt(total) if not math.isnan(total) else math.nan, 0.0
    n = scale * math.sqrt(total)
    return n, scale * min(1.0, max_norm / (n + 1e-6))


def adamw(p, m, v, g, coef, step, lr, betas, eps, decay):
    """(p, m, v) after the update, and a bound of what 32-bit arithmetic may be off by in each."""
    p, m, v, g = (x.cpu().to(F64) for x in (p, m, v, g))
    g = coef * g
    b1, b2 = betas
    m_new = b1 * m + (1 - b1) * g
    v_new = b2 * v + (1 - b2) * g * g
    den = torch.sqrt(v_new / (1 - b2 ** step)) + eps
    rate = lr / (1 - b1 ** step)
    p_new = p - lr * decay * p - rate * m_new / den
    # Each product, sum and rounded constant is off by U of the terms' size: g by one (its product with coef), the two
    # products by three and four, their sum by one more; the moments' terms may cancel, so the bound goes by their sizes.
    size = (b1 * m).abs() + ((1 - b1) * g).abs()
    off_m = 6 * U * size
    off_v = 8 * U * v_new
    # the quotient: numerator as above, denominator half of v's and four roundings, product and difference three
    off_p = 4 * U * p.abs() + 20 * U * rate * size / den
    tiny = 2.0 ** -140            # where a product is below binary32's normal numbers
    return (p_new, m_new, v_new), (off_p + tiny * rate / eps, off_m + tiny, off_v + tiny)


class Policy:
    """Rows of the policy loss in 64 bits: logp, per-row terms, gradient, sums; `off`: a bound of what logp may be off by."""

    def __init__(self, logits, labels, old, adv, weights=None, ref=None, clip=(0.2, 0.2), kl_coef=0.0, temperature=1.0, grad_scale=1.0):
        x = logits.detach().cpu().to(F64)
        rows, vocab = x.shape
        t = 1.0 / temperature
        lab = labels.cpu()
        w = torch.ones(rows, dtype=F64) if weights is None else weights.cpu().to(F64)
        ok = (lab >= 0) & (lab < vocab)
        self.taken = ok & (w != 0)
        self.counts = [int(self.taken.sum()), int(((w != 0) & ~ok).sum())]
        old, adv = old.cpu().to(F64), adv.cpu().to(F64)
        self.logp, self.dlogits, self.off = torch.zeros(rows, dtype=F64), torch.zeros(rows, vocab, dtype=F64), torch.zeros(rows, dtype=F64)
        self.bound = torch.zeros(rows, vocab, dtype=F64)
        sums = [0.0] * 5
        self.sums_off = [0.0] * 5
        for r in torch.nonzero(self.taken).reshape(-1).tolist():
            z = x[r] * t
            top = z.max()
            e = torch.exp(z - top)
            prob = e / e.sum()
            l = z[lab[r]] - top - torch.log(e.sum())
            self.logp[r] = l
            # An exponent is off by 3 U of its size (difference, factor, product), the exponentials' sum by one U for every
            # term that one of at least 64 threads adds and the levels of joining them, the logarithm by a few more of its size.
            spread = float((z[torch.isfinite(z)] - top).abs().mul(prob[torch.isfinite(z)]).sum()) if bool(torch.isfinite(top)) else 0.0
            off = U * (vocab / 64 + 24 + 4 * spread + 4 * abs(float(z[lab[r]] - top)) + 4 * abs(float(torch.log(e.sum()))))
            self.off[r] = off
            rho = torch.exp(l - old[r])
            lo, hi = 1.0 - clip[0], 1.0 + clip[1]
            free, held = -adv[r] * rho, -adv[r] * rho.clamp(lo, hi)
            policy, slope = (free, free) if not free < held else (held, torch.zeros((), dtype=F64))
            cut = float(free < held)
            size = (adv[r] * rho).abs()              # of the slope's terms
            kl = torch.zeros((), dtype=F64)
            if ref is not None:
                d = ref.cpu().to(F64)[r] - l
                kl = torch.exp(d) - d - 1.0
                slope = slope + kl_coef * (1.0 - torch.exp(d))
                size = size + kl_coef * (1.0 + torch.exp(d))
                kl_off = (torch.exp(d) + 1.0) * (off + 4 * U * (1 + abs(float(ref.cpu()[r])))) + 4 * U * (1.0 + d.abs() + torch.exp(d))
            else:
                kl_off = 0.0
            one = torch.zeros(vocab, dtype=F64)
            one[lab[r]] = 1.0
            k = w[r] * grad_scale * t
            self.dlogits[r] = k * slope * (one - prob)
            # the slope is off as its exponentials are; a probability by its exponent and the sum
            slope_off = size * (off + 8 * U + U * (4 + abs(float(l)) + abs(float(old[r]))))
            prob_off = prob * (off + 8 * U + 4 * U * torch.where(torch.isfinite(z), (z - top).abs(), 0.0))
            self.bound[r] = k.abs() * (slope_off * (one + prob) + slope.abs() * (prob_off + 4 * U * (one + prob))) + 2.0 ** -140
            for i, (a, b) in enumerate([(policy + kl_coef * kl, slope_off + kl_coef * kl_off), (policy, slope_off), (kl, kl_off), (cut, 0.0), (1.0, 0.0)]):
                sums[i] += float(w[r] * a)
                self.sums_off[i] += float(w[r].abs() * (b + 4 * U * abs(float(a))))
        self.sums = sums
        self.sums_off = [o + 2 * U * abs(s) for o, s in zip(self.sums_off, sums)]


def half_ulp(x, dtype):
    """What rounding x to the type may change."""
    if dtype == torch.float32:
        return torch.zeros_like(x)
    digits, least = (8, 2.0 ** -133) if dtype == torch.bfloat16 else (11, 2.0 ** -24)
    return x.abs() * 2.0 ** -digits + least / 2
