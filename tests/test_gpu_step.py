"""Global gradient norm, clipping and AdamW over lists of tensors, against their definitions in 64 bits."""
import math

import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PIECE = 4096
# sizes around a piece's end and around a thread's share of it, single elements, tensors without any
SIZES = {"one": [1], "edges": [1, 0, 3, 4, 5, 7, 8, 9, 2047, 2048, 2049, PIECE - 1, 0, PIECE, PIECE + 1, 3 * PIECE + 5, 31, 1025],
         "many": [1 + 37 * i % 911 for i in range(700)], "long": [2 ** 22 + 3, 100003], "none": [0, 0]}
LAYOUTS = ["apart", "packed"]       # every tensor an allocation of its own, or one behind the other from an odd element on
HYPER = dict(step=7, lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def laid(sizes, layout, dtype, make):
    if layout == "apart":
        return [make(n).to(dtype) for n in sizes]
    buf = torch.zeros(sum(sizes) + 8, dtype=dtype, device=DEV)
    out, at = [], 1
    for n in sizes:
        out.append(buf[at:at + n])
        out[-1].copy_(make(n))
        at += n
    return out


def values(seed, scale):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return lambda n: torch.randn(n, device=DEV, generator=gen) * scale


def record():
    return torch.full((2,), 7.0, device=DEV)


def close(got, want, rel):
    return got == want or abs(got - want) <= rel * abs(want)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("sizes", list(SIZES))
def test_norm_and_clip(sizes, dtype, layout):
    numel, kind = SIZES[sizes], R.DTYPES[dtype]
    g = laid(numel, layout, kind, values(1, 0.1))
    to = laid(numel, layout, kind, lambda n: torch.full((n,), 9.0, device=DEV))
    h = S.Step(numel, kind)
    h.bind(grads=g)
    before = [x.clone() for x in g]
    for scale, most in ((1.0, 2.0 ** -7), (0.5, 1e6), (2.0 ** -10, math.inf)):
        out = record()
        h.mc_grad_norm(most, out, scale)
        norm, coef = R.norm(g, scale, most)
        # binary64 up to one rounding of each result
        assert close(float(out[0]), norm, 1.01 * R.U) and close(float(out[1]), coef, 1.01 * R.U), (sizes, scale)
        again = record()
        h.bind(clipped=to)
        h.mc_grad_clip(most, again, scale)
        assert torch.equal(out, again)
        for x, b, y in zip(g, before, to):
            assert torch.equal(x, b) and torch.equal(y, (b.float() * out[1]).to(kind))
        if layout == "packed":
            edge = to[0]._base if to[0]._base is not None else to[0]
            assert float(edge[0]) == 0 and float(edge[-1]) == 0
    h.close()


@pytest.mark.parametrize("dtype", list(R.DTYPES))
def test_clip_in_place(dtype):
    numel, kind = SIZES["edges"], R.DTYPES[dtype]
    g = laid(numel, "packed", kind, values(2, 1.0))
    before = [x.clone() for x in g]
    h, out = S.Step(numel, kind), record()
    h.bind(grads=g)
    h.mc_grad_clip(1.0, out)
    assert float(out[1]) < 0.1
    assert all(torch.equal(x, (b.float() * out[1]).to(kind)) for x, b in zip(g, before))


@pytest.mark.parametrize("scale", [1e30, 1e-30])
def test_squares_beyond_32_bits(scale):
    numel = SIZES["edges"]
    for kind in (torch.float32, torch.bfloat16):
        g = laid(numel, "packed", kind, values(3, scale))
        h, out = S.Step(numel, kind), record()
        h.bind(grads=g)
        h.mc_grad_norm(1.0, out)
        norm, coef = R.norm(g, 1.0, 1.0)
        assert close(float(out[0]), norm, 1.01 * R.U) and close(float(out[1]), coef, 1.01 * R.U)
        assert norm > 0 and math.isfinite(norm)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
def test_not_finite(dtype, bad):
    """No coefficient, zeros where the gradient is clipped, and no update."""
    numel, kind = SIZES["edges"], R.DTYPES[dtype]
    g = laid(numel, "packed", kind, values(4, 0.1))
    g[-3][PIECE + 100] = bad
    to, lists = laid(numel, "packed", kind, values(5, 1.0)), [laid(numel, "packed", torch.float32, values(6 + i, 1.0)) for i in range(3)]
    model = laid(numel, "packed", torch.bfloat16, values(9, 1.0))
    before = [[x.clone() for x in l] for l in (*lists, model)]
    h, out = S.Step(numel, kind, torch.bfloat16), record()
    h.bind(grads=g, clipped=to, params=lists[0], exp_avg=lists[1], exp_avg_sq=lists[2], model=model)
    h.mc_grad_clip(1.0, out)
    assert float(out[1]) == 0.0 and (math.isnan(float(out[0])) if math.isnan(bad) else float(out[0]) == math.inf)
    assert all(bool((x == 0).all()) for x in to)
    h.mc_adamw(coef=out[1:], **HYPER)
    assert all(torch.equal(x, y) for l, m in zip((*lists, model), before) for x, y in zip(l, m))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("copy", ["none", "bf16", "f16"])
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("sizes", ["one", "edges", "many", "none"])
def test_adamw(sizes, dtype, copy, layout):
    numel, kind, to = SIZES[sizes], R.DTYPES[dtype], R.DTYPES.get(copy)
    g = laid(numel, layout, kind, values(11, 0.3))
    p, m = laid(numel, layout, torch.float32, values(12, 0.5)), laid(numel, layout, torch.float32, values(13, 0.1))
    v = laid(numel, layout, torch.float32, lambda n: values(14 + n, 0.1)(n).square())
    lists = dict(grads=g, params=p, exp_avg=m, exp_avg_sq=v)
    still = [i % 3 == 1 for i in range(len(numel))]
    h, out = S.Step(numel, kind, to, no_decay=still), record()
    if to is not None:
        lists["model"] = laid(numel, layout, to, lambda n: torch.zeros(n, device=DEV))
    h.bind(**lists)
    h.mc_grad_norm(1.0, out)
    for coef in (out[1:], None):
        want = [R.adamw(a, b, c, d, 1.0 if coef is None else float(coef), HYPER["step"], HYPER["lr"], HYPER["betas"], HYPER["eps"], 0.0 if s else 0.1)
                for a, b, c, d, s in zip(p, m, v, g, still)]
        h.mc_adamw(coef=coef, **HYPER)
        for t, (exact, off) in enumerate(want):
            for name, got, e, o in zip("pmv", (p[t], m[t], v[t]), exact, off):
                assert bool(((got.cpu().double() - e).abs() <= o).all()), (name, t)
            if to is not None:
                assert torch.equal(lists["model"][t], p[t].to(to))
    if layout == "packed":
        for l in lists.values():
            base = l[0]._base if l[0]._base is not None else l[0]
            assert float(base[0]) == 0 and float(base[-1]) == 0
    h.close()


def test_bound_again():
    """What a list is bound to last counts, for the calls issued afterwards."""
    numel = [5000, 3]
    a, b = (laid(numel, "apart", torch.float32, values(s, 1.0)) for s in (21, 22))
    h, first, second = S.Step(numel), record(), record()
    h.bind(grads=a)
    h.mc_grad_norm(1.0, first)
    h.bind(grads=b)
    h.mc_grad_norm(1.0, second)
    assert close(float(first[0]), R.norm(a, 1, 1)[0], 1.01 * R.U) and close(float(second[0]), R.norm(b, 1, 1)[0], 1.01 * R.U)


def test_on_another_stream():
    numel = SIZES["long"]
    g = laid(numel, "apart", torch.float32, values(23, 1.0))
    h, out = S.Step(numel), record()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for x in g:
            x.mul_(0.5)
        h.bind(grads=g)
        h.mc_grad_norm(1.0, out)
    side.synchronize()
    assert close(float(out[0]), R.norm(g, 1, 1)[0], 1.01 * R.U)


def test_same_bits_every_time():
    numel = SIZES["long"] + SIZES["many"]
    g = laid(numel, "packed", torch.float32, values(24, 1.0))
    h, outs = S.Step(numel), [record() for _ in range(20)]
    h.bind(grads=g)
    for out in outs:
        h.mc_grad_norm(1.0, out)
    assert all(torch.equal(outs[0], o) for o in outs)


def test_more_elements_than_31_bits():
    n = 2 ** 31 + 4099
    x = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    x[-1], x[2 ** 31 - 1], x[0] = 3.0, 4.0, 12.0
    h, out = S.Step([n], torch.bfloat16), record()
    h.bind(grads=[x])
    h.mc_grad_clip(6.5, out)
    assert float(out[0]) == 13.0 and close(float(out[1]), 6.5 / (13.0 + 1e-6), 1.01 * R.U)
    coef = float(out[1])
    assert [float(x[i]) for i in (-1, 2 ** 31 - 1, 0)] == [float(torch.tensor(y * coef).bfloat16()) for y in (3.0, 4.0, 12.0)]
    assert int(torch.count_nonzero(x)) == 3
    h.close()
    del x
    torch.cuda.empty_cache()


def test_refusals():
    def status(call):
        with pytest.raises(B.McError) as e:
            call()
        return e.value.status
    numel = [100, 0, 7]
    g = laid(numel, "apart", torch.float32, values(31, 1.0))
    h, out = S.Step(numel, torch.float32, torch.bfloat16), record()
    assert status(lambda: h.mc_grad_norm(1.0, out)) == B.MC_ERR_INVALID_ARG                 # nothing bound
    h.bind(grads=g)
    for most, scale in ((0.0, 1.0), (-1.0, 1.0), (math.nan, 1.0), (1.0, 0.0), (1.0, math.inf), (1.0, math.nan)):
        assert status(lambda: h.mc_grad_norm(most, out, scale)) == B.MC_ERR_INVALID_ARG
        assert status(lambda: h.mc_grad_clip(most, out, scale)) == B.MC_ERR_INVALID_ARG
    assert status(lambda: h.mc_adamw(**HYPER)) == B.MC_ERR_INVALID_ARG                      # no weights bound
    h.bind(params=g, exp_avg=g, exp_avg_sq=g)
    assert status(lambda: h.mc_adamw(**HYPER)) == B.MC_ERR_INVALID_ARG                      # no copy bound
    h.bind(model=[x.bfloat16() for x in g])
    for wrong in (dict(step=0), dict(lr=-1.0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(weight_decay=math.inf)):
        assert status(lambda: h.mc_adamw(**{**HYPER, **wrong})) == B.MC_ERR_INVALID_ARG, wrong
    for bad in ([g[0], g[1]], [g[0], g[1], g[2].half()], [g[0], g[1], g[2][:6]], [g[0][::2], g[1], g[2]], [g[0].cpu(), g[1], g[2]]):
        with pytest.raises(ValueError):
            h.bind(grads=bad)
    for bad in (torch.empty(3, device=DEV), torch.empty(2), torch.empty(2, device=DEV, dtype=torch.float64)):
        with pytest.raises(ValueError):
            h.mc_grad_norm(1.0, bad)
    with pytest.raises(ValueError):
        S.Step(numel).bind(model=g)
    L, addresses = S.lib(), B.ptr_array(g)
    addresses[2] = g[2].data_ptr() + 2                                                       # off an element's boundary
    assert L.mc_step_bind(h._h, 0, addresses, None) == B.MC_ERR_INVALID_ARG
    addresses[2] = None
    assert L.mc_step_bind(h._h, 0, addresses, None) == B.MC_ERR_INVALID_ARG
    for out_of in (-1, 6):
        assert L.mc_step_bind(h._h, out_of, B.ptr_array(g), None) == B.MC_ERR_INVALID_ARG
    h.mc_grad_norm(1.0, out)                                                                 # refused calls left the handle as it was
    assert close(float(out[0]), R.norm(g, 1, 1)[0], 1.01 * R.U)
