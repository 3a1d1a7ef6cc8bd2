"""Token log-probabilities and the policy loss at the ends of what their arguments may be, against the definitions in 64 bits."""
import math

import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import step as S
from test_gpu_policy_loss import DEV, rows_of, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loss():
    h = S.PolicyLoss()
    yield h
    h.close()


@pytest.mark.parametrize("temperature", [1e-38, 1e-30, 1e-20, 1e-17, 1e-16, 1e-8, 1e8, 1e30, 3e38])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", [5, 600, 9000, 70001, 140001])
def test_any_temperature(loss, vocab, dtype, temperature):
    """From where a row is its largest logit to where all of it is alike; minus infinity stays without a probability."""
    rows = 6
    x, labels, gen = rows_of(rows, vocab, dtype, vocab)
    x[1, 1:], labels[1] = -math.inf, 0
    x[2, vocab // 2:], labels[2] = -math.inf, 1
    x[3] = 0.25
    if temperature < 1.0:
        labels[4:] = x[4:].float().argmax(1).cpu()
        if temperature < 1e-30:                      # the others' log-probabilities would be beyond 32 bits
            labels[:3] = x[:3].float().argmax(1).cpu()
    temperature = float(torch.tensor(temperature))   # as it is handed over
    zero = torch.zeros(rows)
    want = R.Policy(x, labels, zero, zero, temperature=temperature)
    out = torch.full((rows,), 5.0, device=DEV)
    loss.mc_token_logp(x, labels.to(DEV), out, temperature=temperature)
    sums, logp, dx = run(loss, x, labels, want.logp.float().to(DEV), torch.ones(rows, device=DEV), None, None, temperature=temperature, grad_scale=temperature)
    for got in (out, logp):
        # (rounded to 32 bits once more, where the others of the bound's parts are of the same size)
        assert bool(((got.cpu().double() - want.logp).abs() <= want.off + R.U * want.logp.abs()).all()), (got, want.logp)
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(sums[:5]).all())
    assert not bool(dx[1].any()) and not bool(dx[2, vocab // 2:].any())
