"""The operators of a step in few bits together: a layer's gradients, the example's step, and the exchange of gradients between them."""
import os
import sys

import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import mx as X
from paper_2103_15195_amd import step as S

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import lowbit_step as E  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def quantised(x):
    """What a matrix's values stand for after mc_mx_quantize, by rows and by columns, in 64 bits."""
    cols = x.shape[1]
    return R.values4(*R.quantized(x))[:, :cols], R.values4(*R.quantized(x.t()))[:, :x.shape[0]].t()


@pytest.mark.parametrize("shape", [(1, 5, 33), (70, 40, 200), (150, 300, 129)], ids=str)
def test_gradients_of_a_product(shape):
    """Operands and slopes that 4 bits hold exactly: gradients are the formula's to the last bit, and so are differences of the loss, which is linear in either operand."""
    (m, n, k), mx = shape, X.Mx()
    rng = np.random.default_rng(1)
    x, w, dy = (torch.from_numpy(R.GRID[rng.integers(1, 8, s)] * rng.choice([-1.0, 1.0], s)).float().to(DEV) for s in ((m, k), (n, k), (m, n)))
    for t in (x, w, dy):                                     # every block along rows and columns has a 6, and so the scale 1, under which its values are themselves
        t[:, ::32], t[::32, :] = 6.0, 6.0

    def pair(t):
        r, c = X.MxMatrix(*t.shape), X.MxMatrix(t.shape[1], t.shape[0])
        mx.mc_mx_quantize(t, r, c)
        return r, c

    def loss(a, b):
        y = torch.empty(m, n, device=DEV)
        mx.mc_mx_matmul(pair(a)[0], pair(b)[0], y)
        return (quantised(dy.cpu())[0] * y.cpu().double()).sum()
    (xr, xc), (wr, wc), (dr, dc) = pair(x), pair(w), pair(dy)
    dx, dw = torch.empty(m, k, device=DEV), torch.empty(n, k, device=DEV)
    mx.mc_mx_matmul(dr, wc, dx)
    mx.mc_mx_matmul(dc, xc, dw)
    assert torch.equal(dx.cpu().double(), quantised(dy.cpu())[0] @ quantised(w.cpu())[1])
    assert torch.equal(dw.cpu().double(), quantised(dy.cpu())[1].t() @ quantised(x.cpu())[1])
    # an element to another value of the grid: the blocks' largest stay, and so do all other elements
    i, j = m - 1, k - 1
    assert all(bool((q == t.cpu()).all()) for t in (x, w, dy) for q in quantised(t.cpu()))
    other = x.clone()
    other[i, j] = -x[i, j]
    assert float(loss(other, w) - loss(x, w)) == float(dx[i, j].double() * (other[i, j] - x[i, j]).double())
    other = w.clone()
    other[n - 1, j] = -w[n - 1, j]
    assert float(loss(x, other) - loss(x, w)) == float(dw[n - 1, j].double() * (other[n - 1, j] - w[n - 1, j]).double())


def test_a_step_of_the_example():
    """Logits, gradients and the update of one step against the same in 64 bits, layer by layer from what the step itself had in 32 bits."""
    t = E.Training(seed=3)
    x = torch.randn(E.BATCH, E.SIZES[0], device=DEV, generator=t.gen)
    labels = torch.randint(0, E.SIZES[-1], (E.BATCH,), device=DEV, generator=t.gen)
    t.gradients(x, labels)
    inputs = [x] + [torch.relu(l.y) for l in t.layers[:-1]]
    slopes = t.slopes
    bound = 8 * 2.0 ** -23                                   # a matrix instruction's levels and the sum, of each step's terms
    for i in range(len(t.layers) - 1, -1, -1):
        l = t.layers[i]
        xr, xc = quantised(inputs[i].cpu())
        wr, wc = quantised(l.model.cpu())
        dr, dc = quantised(slopes.cpu())
        steps = lambda k: (k + 127) // 128 + 8  # noqa: E731
        assert bool(((l.y.cpu().double() - (xr @ wr.t() + l.bias.cpu().double())).abs() <= bound * steps(xr.shape[1]) * (xr.abs() @ wr.abs().t()) + 1e-30).all())
        assert bool(((l.dweight.cpu().double() - dc.t() @ xc).abs() <= bound * steps(E.BATCH) * (dc.abs().t() @ xc.abs()) + 1e-30).all())
        assert bool(((l.dbias.cpu().double() - slopes.cpu().double().sum(0)).abs() <= E.BATCH * R.U * slopes.cpu().double().abs().sum(0)).all())
        if i:
            assert bool(((l.dx.cpu().double() - dr @ wc).abs() <= bound * steps(dr.shape[1]) * (dr.abs() @ wc.abs()) + 1e-30).all())
            slopes = torch.where(t.layers[i - 1].y > 0, l.dx, 0.0)
    prob = torch.softmax(t.layers[-1].y.double(), 1)
    one = torch.nn.functional.one_hot(labels, E.SIZES[-1]).double()
    torch.testing.assert_close(t.slopes.double(), (prob - one) / E.BATCH, rtol=1e-4, atol=1e-8)
    # the update, of the list as it is bound
    grads = [g for l in t.layers[::-1] for g in (l.dweight.view(-1), l.dbias)]
    params = [p for l in t.layers[::-1] for p in (l.weight.view(-1), l.bias)]
    t.norm_of.mc_grad_norm(E.MAX_NORM, t.norm)
    lists = [t.moments[k] for k in ("exp_avg", "exp_avg_scale", "exp_avg_sq", "exp_avg_sq_scale")]
    want = [R.adamw8(p, a, b, c, d, g, float(t.norm[1]), 1, E.LR, E.BETAS, 1e-8, 0.0 if i % 2 else E.DECAY)
            for i, (p, a, b, c, d, g) in enumerate(zip(params, *lists, grads))]
    t.update.mc_adamw8(1, E.LR, E.BETAS, weight_decay=E.DECAY, coef=t.norm[1:])
    for i, ((p, m, r), (op, om, orr)) in enumerate(want):
        assert bool(((params[i].cpu().double() - p).abs() <= op).all()), i
        assert R.check8(m, om, lists[0][i], lists[1][i].cpu(), False) == "" and R.check8(r, orr, lists[2][i], lists[3][i].cpu(), True) == ""
    for l in t.layers:
        assert torch.equal(l.model, l.weight.bfloat16()) and torch.equal(l.bias_model, l.bias.bfloat16())
    t.close()


def test_the_example_runs():
    history = E.train(steps=5, seed=1)
    assert len(history) == 5 and all(np.isfinite(h).all() for h in history)


def test_between_the_exchange_and_the_model():
    """Gradients of 4-bit products through a group's compression and sum, their norm and the 8-bit update, for three batches."""
    t = E.Training(seed=5)
    flat = [g.view(-1) for l in t.layers[::-1] for g in (l.dweight, l.dbias)]
    numel = [g.numel() for g in flat]
    ctx = B.Context("fp16", numel, B.mc_partition(numel, 1))
    state, payload = (torch.zeros(f(0), dtype=torch.uint8, device=DEV) for f in (ctx.state_bytes, ctx.payload_bytes))
    for it in range(3):
        x = torch.randn(E.BATCH, E.SIZES[0], device=DEV, generator=t.gen)
        t.gradients(x, torch.randint(0, 10, (E.BATCH,), device=DEV, generator=t.gen))
        before = [g.clone() for g in flat]
        ctx.mc_compress(0, 0, it, flat, state, payload)
        ctx.mc_decompress_sum(0, [payload], 1.0, flat)
        if it == 0:                                          # (later ones have what the first left over)
            assert all(torch.equal(g, b.half().float()) for g, b in zip(flat, before))
        t.norm_of.mc_grad_norm(E.MAX_NORM, t.norm)
        weights = [l.weight.clone() for l in t.layers]
        t.update.mc_adamw8(it + 1, E.LR, E.BETAS, weight_decay=E.DECAY, coef=t.norm[1:])
        assert all(bool(torch.isfinite(l.weight).all()) and not torch.equal(l.weight, w) for l, w in zip(t.layers, weights))
    assert ctx.mc_last_device_status() == B.MC_OK
    ctx.close()
    t.close()


def test_a_layer_in_a_graph():
    """Quantisation, products and update captured together and replayed, between eager calls of the same handles."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    mx, m, n, k = X.Mx(), 300, 70, 20000                     # (sums that blocks share: their parts lie in the handle's scratch)
    x, w, dy = (torch.randn(a, b, device=DEV, generator=gen) for a, b in ((m, k), (n, k), (m, n)))
    mats = {name: (X.MxMatrix(*s), X.MxMatrix(s[1], s[0])) for name, s in (("x", (m, k)), ("w", (n, k)), ("dy", (m, n)))}
    y, dx, dw = torch.empty(m, n, device=DEV), torch.empty(m, k, device=DEV), torch.zeros(n, k, device=DEV)
    h = X.Step8([n * k])
    lists = h.moments()
    h.bind(grads=[dw], params=[w], **lists)

    def step():
        for name, t in (("x", x), ("w", w), ("dy", dy)):
            mx.mc_mx_quantize(t, *mats[name])
        mx.mc_mx_matmul(mats["x"][0], mats["w"][0], y)
        mx.mc_mx_matmul(mats["dy"][0], mats["w"][1], dx)
        mx.mc_mx_matmul(mats["dy"][1], mats["x"][1], dw)
        h.mc_adamw8(1, 1e-2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    held = [w, dw, y, dx, *(t for l in lists.values() for t in l)]
    for i in range(3):
        x.mul_(-0.75)
        before = [t.clone() for t in held]
        graph.replay()
        torch.cuda.synchronize()
        after = [t.clone() for t in held]
        for t, b in zip(held, before):
            t.copy_(b)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(t, a) for t, a in zip(held, after)), i
