"""Token log-probabilities and the clipped policy loss with its gradient, against their definitions in 64 bits."""
import math

import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# around a vector load, a wavefront's and a block's share, and well beyond what one block holds
VOCABS = [1, 2, 3, 7, 8, 9, 10, 63, 64, 65, 257, 511, 512, 513, 1000, 2047, 2048, 2049, 4099, 8192, 16385, 32769, 50001, 65537, 131073, 262147]


@pytest.fixture(scope="module")
def loss():
    h = S.PolicyLoss()
    yield h
    h.close()


def rows_of(rows, vocab, dtype, seed, gap=0, shift=0, scale=3.0):
    """Logits in rows that lie `gap` elements apart, the first `shift` elements into a buffer."""
    gen = torch.Generator().manual_seed(seed)
    ld = vocab + gap
    buf = (torch.randn(rows * ld + shift + 1, generator=gen) * scale).to(R.DTYPES[dtype]).to(DEV)
    x = buf[shift:shift + rows * ld].view(rows, ld)[:, :vocab]
    labels = torch.randint(0, vocab, (rows,), generator=gen)
    return x, labels, gen


def inputs(x, labels, gen, kl, masked=True):
    rows = x.shape[0]
    base = torch.log_softmax(x.double().cpu(), 1)[torch.arange(rows), labels.clamp(0, x.shape[1] - 1)]
    # ratios in steps of 0.05 in the logarithm: none within 0.003 of an edge of the clipping used here
    old = (base - 0.05 * torch.randint(-9, 10, (rows,), generator=gen)).float()
    adv = torch.randn(rows, generator=gen)
    w = torch.rand(rows, generator=gen) + 0.1
    if masked:
        w[torch.rand(rows, generator=gen) < 0.3] = 0.0
    ref = (base + 0.3 * torch.randn(rows, generator=gen)).float() if kl else None
    return old.to(DEV), adv.to(DEV), w.to(DEV), None if ref is None else ref.to(DEV)


def run(loss, x, labels, old, adv, w, ref, dx=None, stream=None, **kw):
    rows, vocab = x.shape
    sums, logp = torch.full((8,), 5.0, device=DEV), torch.full((rows,), 5.0, device=DEV)
    if dx is None:
        dx = torch.full((rows, vocab), 5.0, dtype=x.dtype, device=DEV)
    loss.mc_policy_loss(x, labels.to(DEV), old, adv, weights=w, ref_logp=ref, sums=sums, logp=logp, dlogits=dx, stream=stream, **kw)
    return sums, logp, dx


def check(got, want, dtype):
    sums, logp, dx = got
    torch.cuda.synchronize()
    assert bool(((logp.cpu().double() - want.logp).abs() <= want.off).all())
    bound = want.bound + R.half_ulp(want.dlogits, dtype) * 1.01
    far = (dx.cpu().double() - want.dlogits).abs() - bound
    assert bool((far <= 0).all()), (float(far.max()), int(far.argmax()))
    for a, b, o in zip(sums[:5].tolist(), want.sums, want.sums_off):
        assert abs(a - b) <= o, (a, b, o)
    assert sums.view(torch.int32)[5:].tolist() == [*want.counts, 0]


@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_token_logp(loss, vocab, dtype):
    rows = 37 if vocab < 20000 else 5
    for gap, shift in ((0, 0), (3, 1)):
        x, labels, gen = rows_of(rows, vocab, dtype, vocab, gap, shift)
        labels[1], labels[3], labels[4] = -100, vocab, -2 ** 62
        out = torch.full((rows,), 5.0, device=DEV)
        for t in (1.0, 0.7):
            loss.mc_token_logp(x, labels.to(DEV), out, temperature=t)
            want = R.Policy(x, labels, torch.zeros(rows), torch.zeros(rows), temperature=t)
            assert bool(((out.cpu().double() - want.logp).abs() <= want.off).all())
            assert out[1] == 0 and out[3] == 0 and out[4] == 0


@pytest.mark.parametrize("kl", [False, True])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_policy_loss(loss, vocab, dtype, kl):
    rows = 41 if vocab < 20000 else 6
    kw = dict(clip=(0.2, 0.28), kl_coef=0.1 if kl else 0.0, temperature=0.8, grad_scale=64.0)
    for gap, shift in ((0, 0), (5, 3)):
        x, labels, gen = rows_of(rows, vocab, dtype, vocab + 7, gap, shift)
        old, adv, w, ref = inputs(x.double() / 0.8, labels, gen, kl)
        labels[2], w[2] = -100, 0.5
        wide = torch.full((rows, vocab + gap), 5.0, dtype=x.dtype, device=DEV)
        got = run(loss, x, labels, old, adv, w, ref, dx=wide[:, :vocab], **kw)
        check(got, R.Policy(x, labels, old, adv, w, ref, **kw), x.dtype)
        assert bool((wide[:, vocab:] == 5.0).all())              # nothing behind a row


@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", [10, 1000, 32003, 200001])
def test_in_place_and_forward_only(loss, vocab, dtype):
    x, labels, gen = rows_of(9, vocab, dtype, 5, gap=2)
    old, adv, w, ref = inputs(x, labels, gen, True)
    want = run(loss, x, labels, old, adv, w, ref, kl_coef=0.05)
    sums = torch.empty(8, device=DEV)
    loss.mc_policy_loss(x, labels.to(DEV), old, adv, weights=w, ref_logp=ref, kl_coef=0.05, sums=sums)
    assert torch.equal(sums, want[0])
    got = run(loss, x, labels, old, adv, w, ref, dx=x, kl_coef=0.05)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("vocab", [33, 3000, 40000, 150000])
def test_rows_that_take_no_part(loss, vocab, dtype):
    """Whatever their logits hold: a gradient of zeros, and nothing in the sums."""
    x, labels, gen = rows_of(8, vocab, dtype, 6)
    old, adv, w, ref = inputs(x, labels, gen, True, masked=False)
    x[1], x[3, 5], x[5] = math.nan, math.inf, -math.inf
    w[1] = w[3] = 0.0
    labels[5] = -1
    adv[1] = math.nan
    got = run(loss, x, labels, old, adv, w, ref, kl_coef=0.1)
    keep = [0, 2, 4, 6, 7]
    want = R.Policy(x[keep], labels[keep], old[keep], adv[keep], w[keep], ref[keep], kl_coef=0.1)
    check((got[0].clone(), got[1][keep], got[2][keep]), _with_left_out(want, 1), x.dtype)
    for r in (1, 3, 5):
        assert got[1][r] == 0 and not bool(got[2][r].any()) and not bool(torch.isnan(got[2][r]).any())
    w.zero_()
    sums, logp, dx = run(loss, x, labels, old, adv, w, ref, kl_coef=0.1)
    assert not bool(sums.any()) and not bool(logp.any()) and not bool(dx.any())


def _with_left_out(want, many):
    want.counts[1] = many
    return want


@pytest.mark.parametrize("vocab", [40, 5000, 70001, 140001])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
def test_masked_entries(loss, vocab, dtype):
    """Entries of minus infinity, of the type's lowest value, rows with one entry left, rows of nothing but the lowest value."""
    x, labels, gen = rows_of(6, vocab, dtype, 8)
    least = torch.finfo(x.dtype).min
    half = vocab // 2
    x[0, half:], x[1, :half], x[2, half:] = -math.inf, -math.inf, least
    x[3], x[4] = least, -math.inf
    x[4, 17], labels[4] = 1.5, 17
    labels[0], labels[1], labels[2] = 3, vocab - 1, 4
    old, adv, w, ref = inputs(x, labels, gen, True, masked=False)
    check(run(loss, x, labels, old, adv, w, ref, kl_coef=0.1), R.Policy(x, labels, old, adv, w, ref, kl_coef=0.1), x.dtype)
    # a label that its row rules out, and a row that rules out everything: what the definition says
    labels[0] = vocab - 1
    x[5] = -math.inf
    sums, logp, dx = run(loss, x, labels, old, adv, w, None)
    assert logp[0] == -math.inf and math.isnan(float(logp[5])) and math.isnan(float(sums[0]))
    assert bool(torch.isfinite(dx[1:5]).all())


def test_no_rows(loss):
    sums = torch.full((8,), 5.0, device=DEV)
    x, none = torch.empty(0, 100, device=DEV), torch.empty(0, device=DEV)
    loss.mc_policy_loss(x, none.long(), none, none, sums=sums, dlogits=torch.empty_like(x), logp=none)
    assert not bool(sums.any())
    loss.mc_token_logp(x, none.long(), none)


@pytest.mark.parametrize("rows,vocab", [(5000, 17), (20000, 3), (2500, 1100), (3000, 5003)])
def test_many_rows(loss, rows, vocab):
    """More rows than blocks: against the same rows a few at a time."""
    x, labels, gen = rows_of(rows, vocab, "bf16", 9)
    old, adv, w, ref = inputs(x, labels, gen, True)
    sums, logp, dx = run(loss, x, labels, old, adv, w, ref, kl_coef=0.1)
    total, counts = torch.zeros(5, dtype=torch.float64), torch.zeros(2, dtype=torch.int64)
    off = 2 * R.U * (vocab / 64 + 24 + 8 * 30)            # of logp, both ways; logits stay within 30 of each other
    for r in range(0, rows, 999):
        s = slice(r, r + 999)
        a, b, c = run(loss, x[s], labels[s], old[s], adv[s], w[s], ref[s], kl_coef=0.1)
        assert bool(((b - logp[s]).abs() <= off).all())
        assert bool(((c.float() - dx[s].float()).abs() <= c.float().abs() * 2.0 ** -7 + 2.0 ** -100).all())      # a unit in the last place
        total += a[:5].cpu().double()
        counts += a.view(torch.int32)[5:7].cpu()
    assert torch.equal(sums.view(torch.int32)[5:7].cpu().long(), counts)
    # terms add up to less than 3 per row; each part and the whole are rounded once
    assert bool(((sums[:5].cpu().double() - total).abs() <= rows * 3.0 * (4 * R.U + off)).all())


def test_offsets_beyond_32_bits(loss):
    """Rows further apart than 2^31 elements in all."""
    rows, vocab, ld = 3, 70, 2 ** 30 + 11
    buf = torch.empty(2 * ld + vocab, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (rows, vocab), (ld, 1))
    small, labels, gen = rows_of(rows, vocab, "bf16", 10)
    x.copy_(small)
    old, adv, w, ref = inputs(small, labels, gen, True, masked=False)
    check(run(loss, x, labels, old, adv, w, ref, dx=x), R.Policy(small, labels, old, adv, w, ref), x.dtype)
    del buf, x
    torch.cuda.empty_cache()


def test_gradient_against_differences(loss):
    """Along random directions, the 64-bit loss's central difference: off by h^2 / 6 times its third derivative, which stays
    below 40 for logits of this size and directions of length one (the loss's own derivatives are sums of at most
    rows * weight * (|A| rho + kl exp(d)) times the softmax's, which are below one)."""
    x, labels, gen = rows_of(12, 50, "f32", 11, scale=1.0)
    old, adv, w, ref = inputs(x, labels, gen, True)
    kw = dict(clip=(0.2, 0.3), kl_coef=0.2, temperature=1.3)
    _, _, dx = run(loss, x, labels, old, adv, w, ref, **kw)
    h, bound = 2.0 ** -10, R.Policy(x, labels, old, adv, w, ref, **kw).bound
    for k in range(20):
        d = torch.randn(12, 50, generator=gen, dtype=torch.float64)
        d /= d.norm()
        up, down = (R.Policy(x.cpu().double() + s * h * d, labels, old, adv, w, ref, **kw).sums[0] for s in (1, -1))
        assert abs((up - down) / (2 * h) - float((dx.cpu().double() * d).sum())) <= 40 * h * h / 6 + float((bound * d.abs()).sum())


def test_same_bits_and_another_stream(loss):
    x, labels, gen = rows_of(700, 3001, "bf16", 12)
    old, adv, w, ref = inputs(x, labels, gen, True)
    first = run(loss, x, labels, old, adv, w, ref, kl_coef=0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for k in range(5):
        with torch.cuda.stream(side):
            again = run(loss, x, labels, old, adv, w, ref, kl_coef=0.1)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_refusals(loss):
    x, labels, gen = rows_of(4, 30, "f32", 13)
    old, adv, w, ref = inputs(x, labels, gen, True)
    lab, sums, logp = labels.to(DEV), torch.empty(8, device=DEV), torch.empty(4, device=DEV)

    def refused(kind, *a, **k):
        with pytest.raises(kind) as e:
            loss.mc_policy_loss(*a, **{"sums": sums, **k})
        return getattr(e.value, "status", None)
    for k in (dict(temperature=0.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(clip=(-0.1, 0.2)), dict(clip=(1.1, 0.2)),
              dict(clip=(0.2, -0.1)), dict(clip=(0.2, math.inf)), dict(kl_coef=-1.0), dict(kl_coef=math.nan), dict(grad_scale=math.inf)):
        assert refused(B.McError, x, lab, old, adv, **k) == B.MC_ERR_INVALID_ARG, k
    wrong = [(x.double(), lab, old, adv), (x.t(), lab, old, adv), (x, lab.int(), old, adv), (x, lab[:3], old, adv), (x, lab, old[:3], adv),
             (x, lab, old, adv.double()), (x.cpu(), lab, old, adv)]
    for a in wrong:
        refused(ValueError, *a)
    for k in (dict(weights=w[:3]), dict(ref_logp=ref.half()), dict(logp=torch.empty(3, device=DEV)), dict(sums=torch.empty(7, device=DEV)),
              dict(dlogits=torch.empty(4, 29, device=DEV)), dict(dlogits=torch.empty(4, 30, device=DEV).half()), dict(dlogits=torch.empty(30, 4, device=DEV).t())):
        refused(ValueError, x, lab, old, adv, **k)
    with pytest.raises(ValueError):
        loss.mc_token_logp(x, lab, torch.empty(5, device=DEV))
    with pytest.raises(B.McError):
        loss.mc_token_logp(x, lab, logp, temperature=-1.0)
