"""The policy loss's KL term and its slope where the policy is close to its reference: both go to 0 with the distance d of the log-probabilities, the
term as d^2 / 2, and keep their digits.

Rows in which one logit outweighs all others so far that their sum is 1 in 32 bits: the log-probability is then as near to 0 as its logarithm is exact,
and what the call writes of it has all its digits, so that d is known as the kernel has it.  Term and slope are compared with those of this d in 64 bits."""
import math

import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import step as S
from test_gpu_policy_loss import DEV, inputs, rows_of, run

pytestmark = pytest.mark.gpu
# a row by 16 and 64 threads, by blocks of several sizes, by one that holds it in part, shared by blocks
VOCABS = [2, 100, 1000, 5000, 17000, 40000, 70000, 140000]
DISTANCES = [s * 10.0 ** e * f for e in range(-6, 1) for f in (1.0, 2.3, 4.9) for s in (1, -1)] + [0.0]


@pytest.fixture(scope="module")
def loss():
    h = S.PolicyLoss()
    yield h
    h.close()


def term(d):
    """exp(d) - d - 1 in 64 bits: by its series where the difference has lost a third of its digits."""
    if abs(d) > 0.05:
        return math.expm1(d) - d
    return math.fsum(d ** n / math.factorial(n) for n in range(2, 14))


@pytest.mark.parametrize("rows", [1, 140])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_term_and_slope_close_to_the_reference(loss, vocab, dtype, rows):
    x = torch.zeros(rows, vocab, dtype=R.DTYPES[dtype], device=DEV)
    label = vocab // 3
    x[:, label] = 40.0
    labels = torch.full((rows,), label, device=DEV)
    zero = torch.zeros(rows, device=DEV)
    at = rows - 1                                    # the one row that takes part
    w = zero.clone()
    w[at] = 1.0
    for distance in DISTANCES:
        ref = torch.full((rows,), distance, device=DEV)
        sums, logp, dx = run(loss, x, labels, zero, zero, w, ref, kl_coef=1.0, grad_scale=2.0 ** 40)
        l = float(logp[at])
        assert abs(l) <= 2.0 ** -23                  # two units in the last place of log(1/2)
        d = float(ref[at]) - l
        got, want = float(sums[2]), term(d)
        # d rounded to 32 bits, twice as much in its square; a polynomial's or a difference's few, whose operands are at most
        # five times the result; the product with the weight, and the sum's rounding
        assert got >= 0.0 and abs(got - want) <= 16 * R.U * want, (distance, got, want)
        assert float(sums[0]) == got and float(sums[1]) == 0.0
        if dtype == "f32":
            # - slope * exp(-40) anywhere else: an exponent's three roundings, 40 each, and a few of slope and products
            other, slope = float(dx[at, (label + 1) % vocab]), math.expm1(d) * 2.0 ** 40 * math.exp(-40.0)
            assert abs(other - slope) <= 140 * R.U * abs(slope), (distance, other, slope)


@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", [7, 300, 9001, 70001])
def test_sum_of_terms_close_to_the_reference(loss, vocab, dtype):
    """Rows of any logits, whose log-probability is off by some 1e-6: the term by that times its slope."""
    rows = 30
    x, labels, gen = rows_of(rows, vocab, dtype, vocab + 2)
    old, adv, w, _ = inputs(x, labels, gen, False)
    exact = R.Policy(x, labels, old, adv, w)
    for size in (1e-3, 1e-2, 0.1):
        ref = (exact.logp + size * torch.randn(rows, generator=gen)).float().to(DEV)
        sums, _, _ = run(loss, x, labels, old, adv, w, ref, kl_coef=0.5)
        want = off = 0.0
        for r in torch.nonzero(exact.taken).reshape(-1).tolist():
            d, by = float(ref[r].double().cpu() - exact.logp[r]), float(exact.off[r])
            want += float(w[r]) * term(d)
            off += float(w[r]) * (1.1 * abs(math.expm1(d)) * by + by * by + 16 * R.U * term(d))
        assert float(sums[2]) >= 0.0 and abs(float(sums[2]) - want) <= off, (size, float(sums[2]), want, off)
