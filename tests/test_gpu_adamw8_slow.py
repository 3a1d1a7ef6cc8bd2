"""AdamW with moments in 8 bits over many updates: which slow changes of the second moment its nearest rounding follows, and which it does not."""
import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import mx as X

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def roots(code, scale):
    return (R.value8(code) * R.spread(scale, code.numel())).float()


@pytest.mark.parametrize("beta2,moves", [(0.999, False), (0.95, False), (0.85, True)])
def test_roots_without_gradients(beta2, moves):
    """Every code from 8 (2^-6) to the largest in a block whose largest root is held by a gradient of 1, the others without one.  A root falls by 1 - sqrt(beta2) of itself:
    0.05 percent at 0.999 and 2.5 at 0.95, less than half of any code's step (1/32 of it, or 1/30 to 1/18), so that every code stays; 7.8 at 0.85, more than half of any of these codes'
    steps, so that all of them leave the normal numbers."""
    codes = torch.arange(8, 0x7F, dtype=torch.uint8)
    n = codes.numel()
    codes = torch.cat([codes.flip(0), torch.full((128 - n,), 0x40, dtype=torch.uint8)])
    h = X.Step8([128])
    lists = h.moments()
    lists["exp_avg_sq"][0].copy_(codes)
    lists["exp_avg_sq_scale"][0].fill_(1.0 / 448.0)
    g, p = torch.zeros(128, device=DEV), torch.zeros(128, device=DEV)
    g[0] = 1.0
    h.bind(grads=[g], params=[p], **lists)
    for step in range(1, 401):
        h.mc_adamw8(step, 0.0, (0.9, beta2))
    got = lists["exp_avg_sq"][0].cpu()
    assert int(got[0]) == 0x7E and float(lists["exp_avg_sq_scale"][0]) == pytest.approx(1 / 448, rel=1e-3)        # (two units in the last place an update)
    assert bool((got[1:] < 8).all()) if moves else torch.equal(got, codes)
    h.close()


@pytest.mark.parametrize("beta2", [0.95, 0.98])
@pytest.mark.parametrize("size", [0.25, 4.0])
def test_roots_follow_gradients_that_vary(beta2, size):
    """Half of the elements' normal gradients become four times smaller, or larger: 2000 updates later their roots are about the true ones.  (The formulas
    over 8192 elements elsewhere: 5 to 95 percent of the ratios between 0.85 and 1.29, the median between 0.99 and 1.04; a tenth more is allowed.)"""
    n = 128 * 64
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    normal = lambda: torch.randn(n, device=DEV, generator=gen)  # noqa: E731
    own, half = torch.exp(0.5 * normal()), torch.rand(n, device=DEV, generator=gen) < 0.5
    h = X.Step8([n])
    lists = h.moments()
    g, p, true = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    h.bind(grads=[g], params=[p], **lists)
    for step in range(1, 4001):
        if step == 2001:
            own = torch.where(half, size * own, own)
        g.copy_(normal() * own)
        true.mul_(beta2).add_((1.0 - beta2) * g.double().square())
        h.mc_adamw8(step, 0.0, (0.9, beta2))
    ratio = (roots(lists["exp_avg_sq"][0], lists["exp_avg_sq_scale"][0]).double() / true.sqrt().cpu())[half.cpu()].sort()[0]
    low, middle, high = (float(ratio[int(len(ratio) * q)]) for q in (0.05, 0.5, 0.95))
    assert 0.77 < low and 0.9 < middle < 1.14 and high < 1.42, (low, middle, high)
    h.close()
