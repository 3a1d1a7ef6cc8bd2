"""The operators around a data-parallel step's exchange of gradients, as cases that can be timed and checked.

After the exchange: the global norm of the summed gradient over a model's list of tensors, clipping by it, and the AdamW
update that takes the clipping coefficient from device memory.  Before it: the loss that back-propagation starts from, a
clipped policy loss with a KL term over a vocabulary, together with its gradient, and the log-probabilities of given tokens
that such a loss is fed with.

Tensor lists are those of the repository's benchmark configurations, or generic ragged ones; a list's tensors are parts of
one buffer (a gradient bucket), each on a boundary of 128 elements, or packed without gaps.
"""
import math
import random

import torch

own = False                       # the plain forms, or the framework's operators

DEV = "cuda:0"
MODELS = {"mlp": 0, "resnet20": 1, "resnet50": 2, "resnet101": 3, "maskrcnn": 4}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PLACE = 128                       # elements: a boundary of 512 bytes in 32 bits
BETAS, EPS, DECAY, RATE, STEP = (0.9, 0.95), 1e-8, 0.1, 3e-4, 1000
MAX_NORM = 1.0
CLIP, TEMPERATURE, KL = (0.2, 0.28), 0.9, 0.05
LOSS_SCALE = {"f32": 1.0, "bf16": 1.0, "f16": 4096.0}         # binary16 gradients would underflow without one


# ---- the repository's tensor lists, as numbers (reverse forward order) ---------------------------------------------
def _bottleneck(blocks):
    fwd, cin = [64 * 3 * 49, 64, 64], 64
    for stage, many in enumerate(blocks):
        mid = 64 << stage
        for b in range(many):
            fwd += [mid * cin, mid, mid, mid * mid * 9, mid, mid, 4 * mid * mid, 4 * mid, 4 * mid]
            if b == 0:
                fwd += [4 * mid * cin, 4 * mid, 4 * mid]
            cin = 4 * mid
    return fwd


def _model(name):
    if name == "mlp":
        fwd = [784 * 256, 256, 256 * 256, 256, 256 * 10, 10]
    elif name == "resnet20":
        fwd, cin = [16 * 27, 16, 16], 16
        for cout in (16, 32, 64):
            for b in range(3):
                fwd += [cout * cin * 9, cout, cout, cout * cout * 9, cout, cout]
                if b == 0 and cin != cout:
                    fwd += [cout * cin, cout, cout]
                cin = cout
        fwd += [640, 10]
    elif name in ("resnet50", "resnet101"):
        fwd = _bottleneck((3, 4, 6, 3) if name == "resnet50" else (3, 4, 23, 3)) + [1000 * 2048, 1000]
    else:
        fwd = _bottleneck((3, 4, 6, 3))
        for cin in (256, 512, 1024, 2048):
            fwd += [256 * cin, 256]
        fwd += [256 * 256 * 9, 256] * 5 + [3 * 256, 3, 12 * 256, 12]
        fwd += [1024 * 12544, 1024, 1024 * 1024, 1024, 91 * 1024, 91, 364 * 1024, 364]
        fwd += [256 * 256 * 9, 256] * 4 + [256 * 256 * 4, 256, 91 * 256, 91]
    return fwd[::-1]


def _list(name, op, model, dtype="f32", copy="", packed=False, tensors=0, elems=0, shape_seed=0):
    c = dict(op=op, model=model, dtype=dtype, copy=copy, packed=packed, tensors=tensors, elems=elems, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _rows(name, op, rows, vocab, dtype="bf16", pad=0, gap=0, seq=256, ref=True, shape_seed=0):
    c = dict(op=op, rows=rows, vocab=vocab, dtype=dtype, pad=pad, gap=gap, seq=seq, ref=ref, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small convolutional network's norm at every step: nothing but latency
        _list("norm_resnet20", "norm", "resnet20"),
        # the headline model's summed gradient, 161 tensors
        _list("norm_resnet50", "norm", "resnet50"),
        # a large model's gradient in 16 bits, odd tensor sizes without gaps between them
        _list("norm_ragged_bf16", "norm", "ragged", "bf16", packed=True, tensors=291, elems=120000007, shape_seed=1),
        # the smallest list clipped before it is compressed
        _list("clip_mlp", "clip", "mlp"),
        # heavy-tailed gradients, which is what clipping is for
        _list("clip_maskrcnn", "clip", "maskrcnn"),
        # the smallest update: six tensors
        _list("adamw_mlp", "adamw", "mlp"),
        # the headline model's update, everything in 32 bits
        _list("adamw_resnet50", "adamw", "resnet50"),
        # a large model in mixed precision: 16-bit gradients and model, 32-bit weights and moments
        _list("adamw_ragged_bf16", "adamw", "ragged", "bf16", "bf16", tensors=291, elems=160000001, shape_seed=2),
        # scoring a batch of sampled sequences once per rollout, for old_logp and ref_logp
        _rows("logp_32k", "logp", 4096, 32000),
        # a classifier's head trained as a policy, a small batch in 32 bits
        _rows("policy_1000", "policy", 64, 1000, "f32", seq=16),
        # one micro-batch of token-level training, a vocabulary padded to a multiple of 64
        _rows("policy_32k", "policy", 4096, 32064, pad=61),
        # a large odd vocabulary, rows apart in a wider buffer
        _rows("policy_odd", "policy", 2048, 128259, gap=5),
    ]


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        op, seed = rng.choice(["norm", "clip", "adamw", "logp", "policy", "policy"]), rng.randrange(1 << 20)
        if op in ("logp", "policy"):
            vocab = int(10.0 ** rng.uniform(1.0, 5.42)) | rng.choice([0, 1])
            rows = int(10.0 ** rng.uniform(0.0, 4.6))
            c = _rows(None, op, rows, vocab, rng.choice(["f32", "bf16", "bf16", "f16"]), pad=rng.choice([0, 0, min(vocab // 2, rng.randrange(1, 64))]),
                      gap=rng.choice([0, 0, rng.randrange(1, 64)]), seq=rng.choice([1, 16, 200, 1024]), ref=rng.random() < 0.7, shape_seed=seed)
        else:
            model = rng.choice(list(MODELS) + ["ragged"] * 5)
            c = _list(None, op, model, rng.choice(["f32", "bf16", "f16"]), rng.choice(["", "bf16", "f16"]) if op == "adamw" else "", packed=rng.random() < 0.5)
            if model == "ragged":
                c["elems"] = int(10.0 ** rng.uniform(3.0, 8.2)) | 1
                c["tensors"] = max(1, min(int(10.0 ** rng.uniform(0.0, 2.6)), c["elems"] // 8))
                c["shape_seed"] = seed
        if work(c)["bytes"] <= most[op]:
            return c


# ---- sizes ---------------------------------------------------------------------------------------------------------
def _numel(case):
    if case["model"] != "ragged":
        return _model(case["model"])
    rng = random.Random(case["shape_seed"])                 # sizes over three decades, odd ones among them
    share = [10.0 ** rng.uniform(0.0, 3.0) for _ in range(case["tensors"])]
    total = sum(share)
    sizes = [max(1, int(case["elems"] * s / total)) for s in share]
    sizes[rng.randrange(len(sizes))] += max(0, case["elems"] - sum(sizes))
    return sizes


def _places(case, numel):
    """First element of every tensor in its buffer, and the buffer's elements."""
    grain = 1 if case["packed"] else PLACE
    at, off = [], 0
    for n in numel:
        at.append(off)
        off += (n + grain - 1) // grain * grain
    return at, off


def _size(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    if case["op"] in ("logp", "policy"):
        n, taken = case["rows"] * case["vocab"], sum(_taken(case))
        if case["op"] == "logp":
            return {"bytes": taken * case["vocab"] * _size(case["dtype"]) + 12 * case["rows"], "flops": 5 * taken * case["vocab"]}
        return {"bytes": (taken * case["vocab"] + n) * _size(case["dtype"]) + (24 + 4 * case["ref"]) * case["rows"], "flops": 9 * taken * case["vocab"]}
    n, b = sum(_numel(case)), _size(case["dtype"])
    if case["op"] == "norm":
        return {"bytes": n * b + 8, "flops": 2 * n}
    if case["op"] == "clip":
        return {"bytes": 2 * n * b + 8, "flops": 3 * n}
    return {"bytes": n * (b + 24 + (2 if case["copy"] else 0)) + 8, "flops": 18 * n}


# ---- values --------------------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed & 0x7FFFFFFFFFFF)
    return gen


def _normal(gen, shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=gen)


def _gradient(case, numel, gen):
    """One flat buffer with the list's tensors at their places, zero between them."""
    at, whole = _places(case, numel)
    x = _normal(gen, whole)
    if case["model"] == "maskrcnn":                         # Student's t with three degrees of freedom
        c = torch.zeros_like(x)
        for _ in range(3):
            c += _normal(gen, whole).square_()
        x *= (c / 3.0).rsqrt_()
    rng = random.Random(case["shape_seed"] + 1)
    ends = at[1:] + [whole]
    std = torch.tensor([10.0 ** rng.uniform(-3.5, -1.0) for _ in numel], device=DEV)
    gone = torch.tensor([e - a - n for a, n, e in zip(at, numel, ends)], device=DEV)
    have = torch.tensor(numel, device=DEV)
    pieces = torch.stack([std, torch.zeros_like(std)], 1).reshape(-1)
    x *= torch.repeat_interleave(pieces, torch.stack([have, gone], 1).reshape(-1), output_size=whole)
    return x.to(DTYPES[case["dtype"]])


def _parts(flat, at, numel):
    return [flat[a:a + n] for a, n in zip(at, numel)]


def _weights(case, numel, gen):
    """32-bit weights and moments of a run that has been going for a while, at their places."""
    at, whole = _places(case, numel)
    p = _normal(gen, whole).mul_(0.05)
    m = _normal(gen, whole).mul_(1e-3)
    v = _normal(gen, whole).mul_(1e-2).square_().add_(1e-7)
    if not case["packed"]:
        there = torch.zeros(whole + 1, device=DEV)          # +1 where a tensor begins, -1 where it ends
        there.index_add_(0, torch.tensor(at, device=DEV), torch.ones(len(at), device=DEV))
        there.index_add_(0, torch.tensor([a + n for a, n in zip(at, numel)], device=DEV), -torch.ones(len(at), device=DEV))
        there = there.cumsum(0, dtype=torch.float64)[:whole] > 0.5
        for x in (p, m, v):
            x *= there
    return p, m, v


def _taken(case):
    """Which tokens of the batch are the policy's: not the prompts, not the padding behind a sequence, and of every
    eighth sequence none."""
    rng, seq, rows = random.Random(case["shape_seed"]), case["seq"], case["rows"]
    taken = []
    while len(taken) < rows:
        first, last = rng.randrange(0, seq // 4 + 1), seq - rng.randrange(0, seq // 3 + 1)
        empty = len(taken) // seq % 8 == 7
        taken += [not empty and first <= i < last for i in range(seq)]
    return taken[:rows]


def _policy_inputs(case, seed):
    gen = _generator(seed * 1000003 + 17)
    rows, vocab, ld = case["rows"], case["vocab"], case["vocab"] + case["gap"]
    wide = _normal(gen, (rows, ld)).mul_(2.5).to(DTYPES[case["dtype"]])
    logits = wide[:, :vocab]
    if case["pad"]:
        logits[:, vocab - case["pad"]:] = float("-inf")     # places that no token has
    labels = torch.randint(0, vocab - case["pad"], (rows,), device=DEV, generator=gen)
    taken = torch.tensor(_taken(case), device=DEV)
    i = {"logits": logits, "labels": labels, "taken": taken}
    if case["op"] == "logp":
        i["labels"] = torch.where(taken, labels, -100)
        return i
    logp = _log_prob(logits, labels, 1.0 / TEMPERATURE)[0]
    # how far the policy has moved from the one that sampled: in steps of 0.02, none of which lies on an edge of the clipping
    i["old"] = logp - 0.02 * torch.round(_normal(gen, rows) * 8.0)
    i["ref"] = logp + 0.3 * _normal(gen, rows) if case["ref"] else None
    i["advantage"] = _normal(gen, rows)
    i["weight"] = taken.float() / taken.sum().clamp(min=1)
    return i


# ---- what a program has in hand ------------------------------------------------------------------------------------
def prepare(case, seed):
    s = {"case": case}
    if case["op"] in ("logp", "policy"):
        s.update(_policy_inputs(case, seed))
        rows, vocab = case["rows"], case["vocab"]
        s["logp"] = torch.empty(rows, device=DEV)
        if case["op"] == "policy":
            s["slope"] = torch.empty(rows, vocab + case["gap"], dtype=DTYPES[case["dtype"]], device=DEV)[:, :vocab]
            s["sums"] = torch.empty(8, device=DEV)
        if own:
            from paper_2103_15195_amd import step as S
            s["loss"] = S.PolicyLoss()
        return s
    numel, gen = _numel(case), _generator(seed * 1000003 + 5)
    at = _places(case, numel)[0]
    s["grad"] = _gradient(case, numel, gen)
    s["norm"] = torch.empty(2, device=DEV)
    lists = {"grads": _parts(s["grad"], at, numel)}
    if case["op"] == "clip":
        s["clipped"] = torch.zeros_like(s["grad"])
        lists["clipped"] = _parts(s["clipped"], at, numel)
    if case["op"] == "adamw":
        s["p"], s["m"], s["v"] = _weights(case, numel, gen)
        s["t"] = STEP
        for name, key in (("params", "p"), ("exp_avg", "m"), ("exp_avg_sq", "v")):
            lists[name] = _parts(s[key], at, numel)
        if case["copy"]:
            s["model"] = s["p"].to(DTYPES[case["copy"]])
            lists["model"] = _parts(s["model"], at, numel)
    if own:
        from paper_2103_15195_amd import step as S
        s["plan"] = S.Step(numel, DTYPES[case["dtype"]], DTYPES[case["copy"]] if case["copy"] else None)
        s["plan"].bind(**lists)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def _log_prob(x, labels, inv_t):
    """Log-probability of each row's label, the row's exponentials and their sum."""
    z = x.float() * inv_t
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = labels.clamp(min=0)[:, None]
    return (z.gather(1, at) - top - torch.log(total))[:, 0], e, total


def _norm(g, out):
    norm = torch.sqrt((g * g).sum())
    out[0] = norm
    out[1] = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    return out[1]


def run(s):
    return _own(s) if own else _plain(s)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "logp":
        valid = s["labels"] >= 0
        s["logp"].copy_(torch.where(valid, _log_prob(s["logits"], s["labels"], 1.0)[0], 0.0))
        return {"logp": s["logp"]}
    if op == "policy":
        inv_t = 1.0 / TEMPERATURE
        logp, e, total = _log_prob(s["logits"], s["labels"], inv_t)
        a, w = s["advantage"], s["weight"]
        ratio = torch.exp(logp - s["old"])
        held = torch.clamp(ratio, 1.0 - CLIP[0], 1.0 + CLIP[1])
        free = -a * ratio >= -a * held
        policy = torch.where(free, -a * ratio, -a * held)
        slope = torch.where(free, -a * ratio, 0.0)
        kl = torch.zeros_like(policy)
        if s["ref"] is not None:
            d = s["ref"] - logp
            kl = torch.exp(d) - d - 1.0
            slope = slope + KL * (1.0 - torch.exp(d))
        taken = w != 0
        slope = torch.where(taken, w * slope * (inv_t * LOSS_SCALE[case["dtype"]]), 0.0)[:, None]
        dx = e * (-slope / total)
        dx.scatter_add_(1, s["labels"][:, None], slope)
        s["slope"].copy_(dx)
        s["logp"].copy_(torch.where(taken, logp, 0.0))
        policy, kl = torch.where(taken, w * policy, 0.0), torch.where(taken, w * kl, 0.0)
        sums = torch.stack([(policy + KL * kl).sum(), policy.sum(), kl.sum(), torch.where(taken & ~free, w, 0.0).sum(), w.sum()])
        counts = torch.stack([taken.sum(), torch.zeros_like(taken).sum()])
        return {"slope": s["slope"], "logp": s["logp"], "sums": sums, "counts": counts.int()}
    g = s["grad"].float()
    coef = _norm(g, s["norm"])
    if op == "norm":
        return {"norm": s["norm"]}
    if op == "clip":
        s["clipped"].copy_(g * coef)
        return {"norm": s["norm"], "clipped": s["clipped"]}
    s["t"] += 1
    p, m, v = s["p"], s["m"], s["v"]
    g = g * coef
    m.mul_(BETAS[0]).add_(g * (1.0 - BETAS[0]))
    v.mul_(BETAS[1]).add_(g * g * (1.0 - BETAS[1]))
    root = torch.sqrt(v) / math.sqrt(1.0 - BETAS[1] ** s["t"]) + EPS
    p.mul_(1.0 - RATE * DECAY).sub_(m / root * (RATE / (1.0 - BETAS[0] ** s["t"])))
    out = {"norm": s["norm"], "p": p, "m": m, "v": v}
    if case["copy"]:
        out["model"] = s["model"].copy_(p)
    return out


def _own(s):
    case, op = s["case"], s["case"]["op"]
    if op == "logp":
        s["loss"].mc_token_logp(s["logits"], s["labels"], s["logp"])
        return {"logp": s["logp"]}
    if op == "policy":
        s["loss"].mc_policy_loss(s["logits"], s["labels"], s["old"], s["advantage"], weights=s["weight"], ref_logp=s["ref"], clip=CLIP, kl_coef=KL,
                                 temperature=TEMPERATURE, grad_scale=LOSS_SCALE[case["dtype"]], sums=s["sums"], logp=s["logp"], dlogits=s["slope"])
        return {"slope": s["slope"], "logp": s["logp"], "sums": s["sums"][:5], "counts": s["sums"].view(torch.int32)[5:7]}
    if op == "norm":
        s["plan"].mc_grad_norm(MAX_NORM, s["norm"])
        return {"norm": s["norm"]}
    if op == "clip":
        s["plan"].mc_grad_clip(MAX_NORM, s["norm"])
        return {"norm": s["norm"], "clipped": s["clipped"]}
    s["t"] += 1
    s["plan"].mc_grad_norm(MAX_NORM, s["norm"])
    s["plan"].mc_adamw(s["t"], RATE, BETAS, EPS, DECAY, coef=s["norm"][1:])
    out = {"norm": s["norm"], "p": s["p"], "m": s["m"], "v": s["v"]}
    if case["copy"]:
        out["model"] = s["model"]
    return out


# ---- the same in 64 bits -------------------------------------------------------------------------------------------
def exact(case, seed):
    f64 = torch.float64
    if case["op"] in ("logp", "policy"):
        i, rows, block = _policy_inputs(case, seed), case["rows"], max(1, (1 << 27) // case["vocab"])
        inv_t = 1.0 / TEMPERATURE if case["op"] == "policy" else 1.0
        logp = torch.zeros(rows, dtype=f64, device=DEV)
        takes = i["taken"]
        for r in range(0, rows, block):
            z = i["logits"][r:r + block].to(f64) * inv_t
            rest = torch.logsumexp(z, 1)
            mine = z[torch.arange(z.shape[0], device=DEV), i["labels"][r:r + block].clamp(min=0)]
            logp[r:r + block] = torch.where(takes[r:r + block], mine - rest, 0.0)
        if case["op"] == "logp":
            return {"logp": logp}
        rho = (logp - i["old"].to(f64)).exp()
        adv, w = i["advantage"].to(f64), i["weight"].to(f64)
        lo, hi = 1.0 - CLIP[0], 1.0 + CLIP[1]
        cut = ((adv > 0) & (rho > hi)) | ((adv < 0) & (rho < lo))          # where the bound holds the objective
        gain = torch.where(cut, rho.clamp(lo, hi), rho) * adv
        by_logp = torch.where(cut, torch.zeros_like(gain), -gain)
        kl = torch.zeros_like(gain)
        if case["ref"]:
            gap = i["ref"].to(f64) - logp
            kl = gap.exp() - 1.0 - gap
            by_logp = by_logp + KL * (1.0 - gap.exp())
        keep = (w != 0).to(f64)
        kl, gain = torch.where(w != 0, kl, 0.0), torch.where(w != 0, gain, 0.0)
        by_logp = torch.where(w != 0, by_logp * w * (inv_t * LOSS_SCALE[case["dtype"]]), 0.0)
        dx = torch.empty(rows, case["vocab"], dtype=f64, device=DEV)
        for r in range(0, rows, block):
            z = i["logits"][r:r + block].to(f64) * inv_t
            dx[r:r + block] = -torch.softmax(z, 1) * by_logp[r:r + block, None]
        dx[torch.arange(rows, device=DEV), i["labels"]] += by_logp
        loss = (w * (KL * kl - gain)).sum()
        return {"slope": dx, "logp": logp, "sums": torch.stack([loss, -(w * gain).sum(), (w * kl).sum(), (w * cut).sum(), w.sum()]), "counts": None}
    numel, gen = _numel(case), _generator(seed * 1000003 + 5)
    g = _gradient(case, numel, gen).to(f64)
    norm = torch.linalg.vector_norm(g)
    coef = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    out = {"norm": torch.tensor([float(norm), coef], dtype=f64, device=DEV)}
    if case["op"] == "clip":
        out["clipped"] = coef * g
    if case["op"] == "adamw":
        p, m, v = _weights(case, numel, gen)
        here = g * coef
        t = STEP + 1
        m = BETAS[0] * m.to(f64) + (1.0 - BETAS[0]) * here
        v = BETAS[1] * v.to(f64) + (1.0 - BETAS[1]) * here.square()
        root = (v / (1.0 - BETAS[1] ** t)).sqrt() + EPS
        p = p.to(f64) - RATE * (DECAY * p.to(f64) + m / (1.0 - BETAS[0] ** t) / root)
        out.update(p=p, m=m, v=v)
        if case["copy"]:
            out["model"] = p
    return out
