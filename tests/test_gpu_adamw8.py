"""AdamW with moments in 8 bits, against its definition in 64 bits."""
import math

import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import mx as X
from paper_2103_15195_amd import step as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# sizes around the ends of a thread's eight elements, a scale's 128, a block's 2048; single elements, tensors without any
SIZES = {"one": [1], "edges": [1, 0, 7, 8, 9, 127, 128, 129, 255, 2047, 2048, 2049, 3 * 2048 + 131, 31, 0, 1025], "many": [1 + 37 * i % 911 for i in range(300)], "none": [0, 0]}
HYPER = dict(step=7, lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def laid(sizes, layout, make):
    """Tensors of their own, or one behind the other from an odd element on."""
    parts = [make(n) for n in sizes]
    if layout == "apart":
        return parts
    buf = torch.zeros(sum(sizes) + 8, dtype=parts[0].dtype, device=DEV)
    out, at = [], 1
    for x in parts:
        out.append(buf[at:at + x.numel()])
        out[-1].copy_(x)
        at += x.numel()
    return out


class Run:
    """A list in the middle of a training, and its handle."""

    def __init__(self, sizes, dtype=torch.float32, copy=None, layout="apart", seed=1, still=None, size=1.0):
        gen = generator(seed)
        normal = lambda n: torch.randn(n, device=DEV, generator=gen)  # noqa: E731
        code = lambda n: torch.randint(0, 256, (n,), device=DEV, generator=gen, dtype=torch.uint8)  # noqa: E731
        positive = lambda n: torch.rand(n, device=DEV, generator=gen) + 0.1  # noqa: E731
        blocks = [(n + 127) // 128 for n in sizes]
        self.sizes = sizes
        self.g = laid(sizes, layout, lambda n: (0.3 * size * normal(n)).to(dtype))
        self.p = laid(sizes, layout, lambda n: 0.5 * normal(n))
        # any code but a NaN's is one that a moment may hold, roots from 0 up
        self.cm = laid(sizes, layout, lambda n: _finite(code(n)))
        self.cr = laid(sizes, layout, lambda n: _finite(code(n)) & 127)
        self.sm = laid(blocks, layout, lambda n: positive(n) * 1e-4 * size)
        self.sr = laid(blocks, layout, lambda n: positive(n) * 1e-4 * size)
        self.model = None if copy is None else laid(sizes, layout, lambda n: torch.zeros(n, dtype=copy, device=DEV))
        self.still = still or [False] * len(sizes)
        self.h = X.Step8(sizes, dtype, copy, no_decay=still)
        lists = dict(grads=self.g, params=self.p, exp_avg=self.cm, exp_avg_sq=self.cr, exp_avg_scale=self.sm, exp_avg_sq_scale=self.sr)
        if copy is not None:
            lists["model"] = self.model
        self.lists = lists
        self.h.bind(**lists)

    def expected(self, coef, **hyper):
        hyper = {**HYPER, **hyper}
        return [R.adamw8(p, cm, sm, cr, sr, g, coef, hyper["step"], hyper["lr"], hyper["betas"], hyper["eps"], 0.0 if s else hyper["weight_decay"])
                for p, cm, sm, cr, sr, g, s in zip(self.p, self.cm, self.sm, self.cr, self.sr, self.g, self.still)]

    def check(self, expected):
        for t, ((p, m, r), (off_p, off_m, off_r)) in enumerate(expected):
            assert bool(((self.p[t].cpu().double() - p).abs() <= off_p).all()), t
            assert R.check8(m, off_m, self.cm[t], self.sm[t].cpu(), False) == "", t
            assert R.check8(r, off_r, self.cr[t], self.sr[t].cpu(), True) == "", t
            if self.model is not None:
                assert torch.equal(self.model[t], self.p[t].to(self.model[t].dtype))


def _finite(code):
    return torch.where(code % 128 == 127, code - 1, code)


@pytest.mark.parametrize("layout", ["apart", "packed"])
@pytest.mark.parametrize("copy", ["none", "bf16", "f16"])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("sizes", list(SIZES))
def test_update(sizes, dtype, copy, layout):
    numel = SIZES[sizes]
    run = Run(numel, DTYPES[dtype], DTYPES.get(copy), layout, still=[i % 3 == 1 for i in range(len(numel))])
    coef = torch.tensor([0.375], device=DEV)
    for c in (coef, None):
        want = run.expected(1.0 if c is None else float(c))
        run.h.mc_adamw8(coef=c, **HYPER)
        run.check(want)
    if layout == "packed":                                   # nothing beside the tensors is written
        for l in run.lists.values():
            base = l[0]._base if l[0]._base is not None else l[0]
            assert float(base[0]) == 0 and float(base[-1]) == 0
    run.h.close()


def test_a_training_from_its_first_step():
    """From moments of zero, ten steps; the moments that are held stay as near to those in 32 bits as their rounding allows."""
    sizes = [1000, 37]
    gen = generator(5)
    h = X.Step8(sizes)
    moments = h.moments()
    p = [torch.randn(n, device=DEV, generator=gen) for n in sizes]
    g = [torch.zeros(n, device=DEV) for n in sizes]
    h.bind(params=p, grads=g, **moments)
    for step in range(1, 11):
        for x in g:
            x.copy_(torch.randn(x.numel(), device=DEV, generator=gen))
        want = [R.adamw8(a, b, c, d, e, f, 1.0, step, 1e-2, (0.9, 0.999), 1e-8, 0.0) for a, b, c, d, e, f in
                zip(p, moments["exp_avg"], moments["exp_avg_scale"], moments["exp_avg_sq"], moments["exp_avg_sq_scale"], g)]
        h.mc_adamw8(step, 1e-2)
        for t, ((pw, m, r), (op, om, orr)) in enumerate(want):
            assert bool(((p[t].cpu().double() - pw).abs() <= op).all()), (step, t)
            assert R.check8(m, om, moments["exp_avg"][t], moments["exp_avg_scale"][t].cpu(), False) == ""
            assert R.check8(r, orr, moments["exp_avg_sq"][t], moments["exp_avg_sq_scale"][t].cpu(), True) == ""
    h.close()


def test_against_32_bits():
    """One update of moments that 8 bits hold exactly gives the weights of mc_adamw."""
    sizes = [3000, 5]
    run = Run(sizes)
    p = [x.clone() for x in run.p]
    m = [(R.value8(c) * R.spread(s, c.numel())).float().to(DEV) for c, s in zip(run.cm, run.sm)]
    v = [(R.value8(c) * R.spread(s, c.numel())).square().float().to(DEV) for c, s in zip(run.cr, run.sr)]
    other = S.Step(sizes)
    other.bind(grads=run.g, params=p, exp_avg=m, exp_avg_sq=v)
    other.mc_adamw(**HYPER)
    want = run.expected(1.0)
    run.h.mc_adamw8(**HYPER)
    for a, b, (_, (off, _, _)) in zip(run.p, p, want):
        assert bool(((a - b).abs().cpu().double() <= 2 * off).all())


def test_a_step_that_is_left_out():
    run = Run(SIZES["edges"], torch.bfloat16, torch.bfloat16)
    run.g[3][2] = math.inf
    before = {k: [x.clone() for x in l] for k, l in run.lists.items()}
    norm, out = S.Step(run.sizes, torch.bfloat16), torch.empty(2, device=DEV)
    norm.bind(grads=run.g)
    norm.mc_grad_norm(1.0, out)
    run.h.mc_adamw8(coef=out[1:], **HYPER)
    assert all(torch.equal(x, y) for k in before for x, y in zip(before[k], run.lists[k]))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_not_finite(bad):
    """An infinity or a NaN stays in its own place: the rest of its block is held as if it were not there."""
    run = Run([2048 + 300])
    run.g[0][130] = bad
    run.g[0][2300] = bad
    want = run.expected(1.0)
    run.h.mc_adamw8(**HYPER)
    (p, m, r), (op, om, orr) = want[0]
    assert not torch.isfinite(m[130]) and not torch.isfinite(m[2300])
    assert R.check8(m, torch.nan_to_num(om, posinf=0.0), run.cm[0], run.sm[0].cpu(), False) == ""
    assert R.check8(r, torch.nan_to_num(orr, posinf=0.0), run.cr[0], run.sr[0].cpu(), True) == ""
    there = torch.ones(p.numel(), dtype=torch.bool)
    there[[130, 2300]] = False
    assert bool(((run.p[0].cpu().double() - p).abs()[there] <= op[there]).all())
    assert bool((int(run.cm[0][130]) & 127 == 127) and (int(run.cr[0][130]) & 127 == 127))


@pytest.mark.parametrize("size", [1e-34, 1e-28, 1e15])
def test_very_small_and_very_large(size):
    """Blocks below 2^-100 are held as zeros, the others with all their digits."""
    run = Run(SIZES["edges"], size=size)
    want = run.expected(1.0)
    run.h.mc_adamw8(**HYPER)
    for t, ((p, m, r), (op, om, orr)) in enumerate(want):
        assert R.check8(m, om, run.cm[t], run.sm[t].cpu(), False) == ""
        if size > 1e-30:                 # (below, squares are no normal numbers of 32 bits)
            assert R.check8(r, orr, run.cr[t], run.sr[t].cpu(), True) == ""
        else:
            assert int(run.cr[t].sum()) == 0 and float(run.sr[t].sum()) == 0


def test_roots_are_never_rounded_to_zero():
    """A gradient 10^5 times as small as its block's largest."""
    n = 256
    h = X.Step8([n])
    lists = h.moments()
    g = torch.full((n,), 1e-6, device=DEV)
    g[0], g[n - 1], g[5] = 1.0, 1.0, 0.0
    p = torch.zeros(n, device=DEV)
    h.bind(grads=[g], params=[p], **lists)
    h.mc_adamw8(1, 1e-3)
    codes = lists["exp_avg_sq"][0].cpu().tolist()
    assert codes[5] == 0 and codes[0] == codes[n - 1] == 0x7E and all(c == 1 for i, c in enumerate(codes) if i not in (0, 5, n - 1))


def test_more_elements_than_31_bits():
    n = 2 ** 31 + 2049
    g, p = torch.zeros(n, dtype=torch.bfloat16, device=DEV), torch.zeros(n, device=DEV)
    h = X.Step8([n], torch.bfloat16)
    lists = h.moments()
    at = [0, 2 ** 31 - 1, 2 ** 31, n - 1]
    for i in at:
        g[i] = 1.0
    h.bind(grads=[g], params=[p], **lists)
    h.mc_adamw8(1, 0.5)
    assert [float(p[i]) for i in at] == pytest.approx([-0.5] * 4, rel=1e-6) and int(torch.count_nonzero(p)) == 4
    assert [int(lists["exp_avg"][0][i]) for i in at] == [0x7E] * 4 and int(torch.count_nonzero(lists["exp_avg_scale"][0])) == len({i // 128 for i in at})
    h.close()
    del g, p, lists
    torch.cuda.empty_cache()


def test_on_a_stream_and_in_a_graph():
    """On a stream of one's own; captured once and replayed, the same as calls one after the other."""
    sizes = SIZES["edges"]
    a, b = Run(sizes, torch.bfloat16, torch.bfloat16, seed=3), Run(sizes, torch.bfloat16, torch.bfloat16, seed=3)
    coef = torch.tensor([0.5], device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.h.mc_adamw8(coef=coef, **HYPER)
    for i in range(3):
        for x, y in zip(a.g, b.g):
            x.mul_(0.75)
            y.mul_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        b.h.mc_adamw8(coef=coef, stream=side, **HYPER)
        side.synchronize()
        assert all(torch.equal(x, y) for k in a.lists for x, y in zip(a.lists[k], b.lists[k])), i


def test_refusals():
    def status(call):
        with pytest.raises(B.McError) as e:
            call()
        return e.value.status
    run = Run([200, 0, 7], torch.float32, torch.bfloat16)
    bare = X.Step8([200, 0, 7])
    assert status(lambda: bare.mc_adamw8(**HYPER)) == B.MC_ERR_INVALID_ARG                     # nothing bound
    for wrong in (dict(step=0), dict(lr=-1.0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(eps=1e-60), dict(weight_decay=math.inf)):
        assert status(lambda: run.h.mc_adamw8(**{**HYPER, **wrong})) == B.MC_ERR_INVALID_ARG, wrong
    for name, l in run.lists.items():
        for bad in (l[:2], [l[0], l[1], l[2].double()], [l[0], l[1], l[0]], [l[0].cpu(), l[1], l[2]]):
            with pytest.raises(ValueError):
                run.h.bind(**{name: bad})
    for bad in (torch.empty(2, device=DEV), torch.empty(1), torch.empty(1, device=DEV, dtype=torch.float64)):
        with pytest.raises(ValueError):
            run.h.mc_adamw8(coef=bad, **HYPER)
    with pytest.raises(ValueError):
        bare.bind(model=run.model)
    with pytest.raises(ValueError):
        X.Step8([1], "float32", "float32")
