"""Policy loss and token log-probabilities where the kernels change form by the number of rows: long rows of which each has a block to itself,
rows whose terms a kernel of its own adds up, more rows than it has room for at a time.  Against the definitions in 64 bits."""
import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import step as S
from test_gpu_policy_loss import DEV, check, inputs, rows_of, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loss():
    h = S.PolicyLoss()
    yield h
    h.close()


# 16-byte vectors of a row held by 1024 threads: 4 or 8 each (32768 and 65536 elements of 16 bits, half as many of 32), 16, more than that
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("vocab,dtype", [(30001, "bf16"), (65530, "f16"), (70001, "bf16"), (131072, "bf16"), (131073, "f16"), (140003, "bf16"), (200001, "bf16"),
                                         (16001, "f32"), (33001, "f32"), (65537, "f32"), (100003, "f32")])
def test_long_rows(loss, vocab, dtype, in_place):
    """More of them than are shared by blocks.  Most take no part, so that the definition has few to go through."""
    rows, kw = 133, dict(kl_coef=0.1, temperature=0.9, grad_scale=16.0)
    x, labels, gen = rows_of(rows, vocab, dtype, vocab + 1, gap=3, shift=5)
    base = x[::11].clone()
    old, adv, w, ref = inputs(x.float()[:, :1].expand(rows, 1), torch.zeros(rows, dtype=torch.int64), gen, True, masked=False)
    some = torch.zeros(rows, dtype=torch.bool)
    some[::11] = True
    w = torch.where(some.to(DEV), w, 0.0)
    picked = inputs(base.double() / 0.9, labels[some], gen, True, masked=False)
    old[some.to(DEV)], ref[some.to(DEV)] = picked[0], picked[3]
    want = R.Policy(base, labels[some], old[some.to(DEV)], adv[some.to(DEV)], w[some.to(DEV)], ref[some.to(DEV)], **kw)
    alone = torch.empty(rows, device=DEV)
    loss.mc_token_logp(x, labels.to(DEV), alone, temperature=0.9)
    got = run(loss, x, labels, old, adv, w, ref, dx=x if in_place else None, **kw)
    some = some.to(DEV)
    check((got[0], got[1][some], got[2][some]), want, x.dtype)
    assert not bool(got[1][~some].any()) and not bool(got[2][~some].any())
    assert bool(((alone[some].cpu().double() - want.logp).abs() <= want.off).all())


@pytest.mark.parametrize("rows,vocab,dtype", [(1500, 37, "f32"), (5000, 20, "bf16"), (1100, 700, "f16"), (300, 9001, "bf16")])
def test_sums_by_a_kernel_of_their_own(loss, rows, vocab, dtype):
    kw = dict(clip=(0.1, 0.3), kl_coef=0.2)
    x, labels, gen = rows_of(rows, vocab, dtype, rows, gap=1)
    old, adv, w, ref = inputs(x, labels, gen, True)
    labels[7], labels[rows - 1] = vocab, -1
    check(run(loss, x, labels, old, adv, w, ref, **kw), R.Policy(x, labels, old, adv, w, ref, **kw), x.dtype)


def test_more_rows_than_terms(loss):
    """300 011 rows are taken in three parts.  The definition for all rows at once; logits of at most 8 in size, five of them: an
    exponent's 3 U of its size, up to 16 / 0.9, the sum's and the logarithm's few, make less than 80 U of the log-probability."""
    rows, vocab, t = 300011, 5, 0.9
    gen = torch.Generator().manual_seed(3)
    x = (torch.randn(rows, vocab, generator=gen) * 2).clamp(-8, 8)
    labels = torch.randint(0, vocab, (rows,), generator=gen)
    labels[::1001] = 5
    valid = labels < vocab
    z = x.double() / t
    prob = torch.softmax(z, 1)
    logp = torch.log_softmax(z, 1)[torch.arange(rows), labels.clamp(max=4)]
    old = (logp - 0.05 * torch.randint(-9, 10, (rows,), generator=gen)).float()
    adv, w = torch.randn(rows, generator=gen), torch.rand(rows, generator=gen)
    w[torch.rand(rows, generator=gen) < 0.3] = 0.0
    on = valid & (w != 0)
    rho = torch.exp(logp - old.double())
    free, held = -adv.double() * rho, -adv.double() * rho.clamp(0.8, 1.2)
    is_free = free >= held
    value, slope = torch.where(is_free, free, held), torch.where(is_free, free, 0.0)
    k = torch.where(on, w.double() * slope / t, 0.0)[:, None]
    dx = -k * prob
    dx[torch.arange(rows), labels.clamp(max=4)] += k[:, 0]
    out = torch.empty(rows, device=DEV)
    xd = x.to(DEV)
    loss.mc_token_logp(xd, labels.to(DEV), out, temperature=t)
    off = 80 * R.U
    assert bool(((out.cpu().double() - torch.where(valid, logp, 0.0)).abs() <= off).all())
    sums, got, slopes = run(loss, xd, labels, old.to(DEV), adv.to(DEV), w.to(DEV), None, temperature=t)
    assert bool(((got.cpu().double() - torch.where(on, logp, 0.0)).abs() <= off).all())
    # the ratio is off as its logarithm is, a probability too, and products by a few U
    size = (w.double() * adv.double().abs() * torch.maximum(rho, held.abs() / adv.double().abs().clamp(min=1e-30)) / t)[:, None]
    assert bool(((slopes.cpu().double() - dx).abs() <= size * (3 * off + 32 * R.U)).all())
    wd = torch.where(on, w.double(), 0.0)
    want = [(wd * value).sum(), (wd * value).sum(), 0.0, (wd * ~is_free).sum(), wd.sum()]
    most = float(size.sum()) * t * (off + 32 * R.U)
    for a, b, o in zip(sums[:5].tolist(), want, (most, most, 0.0, 0.0, 0.0)):
        assert abs(a - float(b)) <= o + 2 * R.U * abs(float(b))
    assert sums.view(torch.int32)[5:].tolist() == [int(on.sum()), int((~valid & (w != 0)).sum()), 0]
