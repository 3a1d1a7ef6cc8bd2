"""A training step in few bits, as cases that can be timed and checked: AdamW with its moments held in 8 bits, matrices
quantised to microscaled 4-bit floating point, and products of such matrices, forward, backward and for single tokens.

Moments: blocks of 128 elements of a tensor, 8-bit floats (four exponent and three mantissa bits) times a 32-bit scale, the second moment
as its root.  Matrices: blocks of 32 elements along a row, each element one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times
a power of two held in 8 bits.  Codes and scales lie in tiles of 16 rows by 128 columns and 64 rows by 128 columns (see `_tiled`).

Tensor lists and some of the matrices are those of the repository's benchmark configurations, the rest is generic.
"""
import math
import random

import torch

own = False                       # the plain forms, or the framework's operators

DEV = "cuda:0"
MODELS = {"mlp": 0, "resnet20": 1, "resnet50": 2, "resnet101": 3, "maskrcnn": 4}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK8, BLOCK4, STEP_K = 128, 32, 128
TOP8, LEAST8, LEAST_AMAX = 448.0, 2.0 ** -9, 2.0 ** -100
BETAS, EPS, DECAY, RATE, STEP = (0.9, 0.95), 1e-8, 0.1, 3e-4, 1000


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


def _list(name, model, dtype="f32", copy="", tensors=0, elems=0, shape_seed=0):
    c = dict(op="adamw8", model=model, dtype=dtype, copy=copy, tensors=tensors, elems=elems, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _matrix(name, op, m, n, k, dtype="bf16", bias=False, gap=0):
    """m rows of k elements, against n rows of weights (quantize: n is 0); dtype: that of the rows and of what comes out."""
    c = dict(op=op, m=m, n=n, k=k, dtype=dtype, bias=bias, gap=gap)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest update, six tensors: nothing but latency
        _list("adamw8_mlp", "mlp"),
        # the headline model's update, gradients and weights in 32 bits
        _list("adamw8_resnet50", "resnet50"),
        # a large model in mixed precision: 16-bit gradients and model, 32-bit weights
        _list("adamw8_ragged_bf16", "ragged", "bf16", "bf16", tensors=291, elems=160000001, shape_seed=2),
        # one token's activations on their way into a product
        _matrix("quantize_token", "quantize", 1, 0, 4096),
        # an odd matrix in 32 bits, rows apart in a wider buffer
        _matrix("quantize_odd", "quantize", 1003, 0, 2049, "f32", gap=3),
        # a large layer's weights, rounded for quantisation-aware training
        _matrix("quantize_weights", "quantize", 8192, 0, 8192),
        # one token's logits over a padded vocabulary: the weights are read once
        _matrix("product_token", "product", 1, 32064, 4096),
        # the detection model's box head, few outputs of a long sum
        _matrix("product_box_head", "product", 512, 1024, 12544, bias=True),
        # a micro-batch's logits, as the policy loss reads them
        _matrix("product_logits", "product", 4096, 32064, 4096),
        # a layer over a small batch of tokens that are being sampled: activations quantised, then multiplied
        _matrix("linear_decode", "linear", 16, 12800, 4096, bias=True),
        # the perceptron's first layer, backward, in 32 bits
        _matrix("backward_mlp", "backward", 256, 256, 784, "f32"),
        # a large layer, backward: gradients of inputs and weights
        _matrix("backward_tokens", "backward", 4096, 8192, 4096),
    ]


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = tuple(max(a, w[k]) for a, k in zip(most.get(c["op"], (0, 0)), ("bytes", "flops")))
    while True:
        op = rng.choice(["adamw8", "quantize", "product", "product", "linear", "backward"])
        if op == "adamw8":
            c = _list(None, rng.choice(list(MODELS) + ["ragged"] * 5), rng.choice(["f32", "bf16", "f16"]), rng.choice(["", "bf16", "f16"]))
            if c["model"] == "ragged":
                c["elems"] = int(10.0 ** rng.uniform(3.0, 8.2)) | 1
                c["tensors"] = max(1, min(int(10.0 ** rng.uniform(0.0, 2.6)), c["elems"] // 8))
                c["shape_seed"] = rng.randrange(1 << 20)
        else:
            size = lambda lo, hi: max(1, int(10.0 ** rng.uniform(lo, hi)) + rng.choice([0, 0, 1]))  # noqa: E731
            few = op == "linear" or (op == "product" and rng.random() < 0.4)
            c = _matrix(None, op, size(0.0, 1.5) if few else size(0.0, 4.0), 0 if op == "quantize" else size(0.7, 4.5), size(1.0, 4.15),
                        rng.choice(["f32", "bf16", "bf16", "f16"]), bias=op in ("product", "linear") and rng.random() < 0.5, gap=rng.choice([0, 0, rng.randrange(1, 64)]))
        w = work(c)
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1]:
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


def _places(numel):
    """First element of every tensor in its buffer, on a boundary of 128 elements, and the buffer's elements."""
    at, off = [], 0
    for n in numel:
        at.append(off)
        off += (n + BLOCK8 - 1) // BLOCK8 * BLOCK8
    return at, off


def _size(dtype):
    return 4 if dtype == "f32" else 2


def _held(rows, cols):
    """Bytes of a quantised matrix: codes and scales."""
    return rows * cols / 2 + rows * math.ceil(cols / BLOCK4)


def work(case):
    if case["op"] == "adamw8":
        n = sum(_numel(case))
        return {"bytes": int(n * (_size(case["dtype"]) + 12.125 + (2 if case["copy"] else 0))) + 4, "flops": 24 * n}
    m, n, k, b = case["m"], case["n"], case["k"], _size(case["dtype"])
    if case["op"] == "quantize":
        return {"bytes": int(2 * m * k * b + _held(m, k)), "flops": 4 * m * k}
    if case["op"] == "product":
        return {"bytes": int(_held(m, k) + _held(n, k) + m * n * b + 4 * n * case["bias"]), "flops": 2 * m * n * k}
    if case["op"] == "linear":
        return {"bytes": int(m * k * b + _held(n, k) + m * n * b + 4 * n * case["bias"]), "flops": 2 * m * n * k}
    return {"bytes": int(m * n * b + _held(k, n) + _held(k, m) + m * k * b + 4 * n * k), "flops": 4 * m * n * k}


# ---- values --------------------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed & 0x7FFFFFFFFFFF)
    return gen


def _normal(gen, shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=gen)


def _list_inputs(case, seed):
    """Gradients, weights and moments of a run that has been going for a while, at their places, zero between them."""
    gen, numel = _generator(seed * 1000003 + 5), _numel(case)
    at, whole = _places(numel)
    rng = random.Random(case["shape_seed"] + 1)
    ends = at[1:] + [whole]
    std = torch.tensor([10.0 ** rng.uniform(-3.5, -1.0) for _ in numel], device=DEV)
    have, gone = torch.tensor(numel, device=DEV), torch.tensor([e - a - n for a, n, e in zip(at, numel, ends)], device=DEV)
    spread = torch.repeat_interleave(torch.stack([std, torch.zeros_like(std)], 1).reshape(-1), torch.stack([have, gone], 1).reshape(-1), output_size=whole)
    there = (spread != 0).float()
    g = (_normal(gen, whole) * spread).to(DTYPES[case["dtype"]])
    p = _normal(gen, whole).mul_(0.05).mul_(there)
    m = _normal(gen, whole).mul_(spread).mul_(0.3)
    root = _normal(gen, whole).mul_(0.3).add_(1.0).abs_().mul_(spread)
    m, ms = _to8(m.view(-1, BLOCK8), False)
    root, rs = _to8(root.view(-1, BLOCK8), True)
    coef = torch.rand(1, device=DEV, generator=gen) * 0.5 + 0.5
    return {"g": g, "p": p, "m": m.view(-1), "ms": ms, "r": root.view(-1), "rs": rs, "coef": coef}


def _rows(gen, rows, cols, dtype, gap, outliers):
    """Rows of activations or of gradients: every column has a size of its own, some are far larger than the rest."""
    wide = _normal(gen, (rows, cols + gap))
    size = torch.exp(0.5 * _normal(gen, cols + gap))
    if outliers:
        size = torch.where(torch.rand(cols + gap, device=DEV, generator=gen) < 0.01, size * 20.0, size)
    return wide.mul_(size).to(DTYPES[dtype])[:, :cols]


def _matrix_inputs(case, seed):
    gen = _generator(seed * 1000003 + 17)
    op, m, n, k, dtype = case["op"], case["m"], case["n"], case["k"], case["dtype"]
    i = {"bias": 0.1 * _normal(gen, n) if case["bias"] else None}
    if op == "quantize":
        return {"x": _rows(gen, m, k, dtype, case["gap"], True)}
    weights = _normal(gen, (n, k)).mul_(k ** -0.5)
    if op == "backward":                                    # of y = x W^T: W and x as the forward pass has laid them out, dy
        i["w"] = _to4(weights.t())
        i["x"] = _to4(_rows(gen, m, k, dtype, 0, True).t())
        i["dy"] = _rows(gen, m, n, dtype, case["gap"], False).mul_(1e-2)
        return i
    i["w"] = _to4(weights)
    x = _rows(gen, m, k, dtype, case["gap"], True)
    i["x"] = _to4(x) if op == "product" else x
    return i


# ---- the plain forms' pieces ---------------------------------------------------------------------------------------
def _to8(x, root):
    """Blocks of 32-bit values as 8-bit floats times a scale."""
    top = x.abs().amax(1)
    scale = torch.where(top >= LEAST_AMAX, top * (1.0 / TOP8), 0.0)
    back = torch.where(scale > 0, 1.0 / scale, 0.0)[:, None]
    code = (x * back).to(torch.float8_e4m3fn)
    if root:                                                # what divides is never rounded to zero
        code = torch.where((x > 0) & (back > 0) & (code.float() == 0), LEAST8, code.float()).to(torch.float8_e4m3fn)
    return code, scale


def _two(e):
    """2^e in 32 bits for whole numbers from -127 to 127, by its bits (a power function need not be exact)."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _round4(x):
    """Values (a multiple of 32 in a row) as multiples of 0.5 up to 6, and the exponents of their blocks' scales."""
    blocks = x.float().reshape(x.shape[0], -1, BLOCK4)
    fraction, exponent = torch.frexp(blocks.abs().amax(2))
    e = torch.where(fraction == 0, -127, exponent - torch.where(fraction <= 0.875, 3, 2)).clamp(-127, 127)
    y = blocks * _two(-e)[:, :, None]
    a = y.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), y), e


def _padded(x):
    rows, cols = x.shape
    out = torch.zeros(rows, math.ceil(cols / STEP_K) * STEP_K, dtype=x.dtype, device=x.device)
    out[:, :cols] = x
    return out


def _tiled(codes, scales):
    """Codes and scales where the products look for them: of 16 rows by 128 columns the 64 pieces of 32 codes, four columns of pieces of 16
    rows each; of 64 rows by 128 columns the scales of each such piece in four sets of 16 rows."""
    rows, steps = codes.shape[0], codes.shape[1] * 2 // STEP_K
    c = torch.zeros((rows + 15) // 16 * 16, steps * 64, dtype=torch.uint8, device=codes.device)
    c[:rows] = codes
    s = torch.zeros((rows + 63) // 64 * 64, steps * 4, dtype=torch.uint8, device=codes.device)
    s[:rows] = scales
    return c.view(-1, 16, steps, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1), s.view(-1, 4, 16, steps, 4).permute(0, 3, 4, 2, 1).contiguous().view(-1)


def _to4(x):
    """A quantised matrix: codes, scales, rows, columns."""
    q, e = _round4(_padded(x))
    a = q.abs()
    code = torch.where(a < 2.0, a * 2.0, torch.where(a < 4.0, a + 2.0, a * 0.5 + 4.0)).to(torch.uint8)     # 0 0.5 1 1.5 2 3 4 6
    code = (code | (torch.signbit(q).to(torch.uint8) << 3)).reshape(x.shape[0], -1)
    codes, scales = _tiled(code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8))
    return {"codes": codes, "scales": scales, "rows": x.shape[0], "cols": x.shape[1]}


GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _from4(q):
    """The values of a quantised matrix, with its columns' padding."""
    rows, steps = q["rows"], (q["cols"] + STEP_K - 1) // STEP_K
    c = q["codes"].view(-1, steps, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(-1, steps * 64)[:rows]
    s = q["scales"].view(-1, steps, 4, 16, 4).permute(0, 4, 3, 1, 2).reshape(-1, steps * 4)[:rows]
    grid = torch.tensor(GRID + [-v for v in GRID], device=DEV)
    x = torch.stack([grid[(c & 15).int()], grid[(c >> 4).int()]], 2).reshape(rows, -1, BLOCK4)
    return (x * _two(s.int() - 127)[:, :, None]).reshape(rows, -1)


def _times(a, b):
    return _from4(a) @ _from4(b).t()


# ---- what a program has in hand ------------------------------------------------------------------------------------
def prepare(case, seed):
    op, s = case["op"], {"case": case}
    if op == "adamw8":
        s.update(_list_inputs(case, seed))
        s["t"] = STEP
        if case["copy"]:
            s["model"] = s["p"].to(DTYPES[case["copy"]])
        if own:
            from paper_2103_15195_amd import mx as X
            numel = _numel(case)
            at = _places(numel)[0]
            many = [(n + BLOCK8 - 1) // BLOCK8 for n in numel]
            first = [a // BLOCK8 for a in at]
            lists = {name: [s[key].view(kind)[a:a + n] for a, n in zip(at, numel)] for name, key, kind in
                     (("grads", "g", s["g"].dtype), ("params", "p", s["p"].dtype), ("exp_avg", "m", torch.uint8), ("exp_avg_sq", "r", torch.uint8))}
            lists.update({name: [s[key][a:a + n] for a, n in zip(first, many)] for name, key in (("exp_avg_scale", "ms"), ("exp_avg_sq_scale", "rs"))})
            if case["copy"]:
                lists["model"] = [s["model"][a:a + n] for a, n in zip(at, numel)]
            s["plan"] = X.Step8(numel, DTYPES[case["dtype"]], DTYPES[case["copy"]] if case["copy"] else None)
            s["plan"].bind(**lists)
        return s
    s.update(_matrix_inputs(case, seed))
    m, n, k, kind = case["m"], case["n"], case["k"], DTYPES[case["dtype"]]
    if op == "quantize":
        s["values"] = torch.empty(m, k, dtype=kind, device=DEV)
    elif op == "backward":
        s["dx"], s["dw"] = torch.empty(m, k, dtype=kind, device=DEV), torch.empty(n, k, device=DEV)
    else:
        s["y"] = torch.empty(m, n, dtype=kind, device=DEV)
    if own:
        from paper_2103_15195_amd import mx as X
        s["mx"] = X.Mx()
        for key in ("w", "x"):
            if isinstance(s.get(key), dict):
                q = s[key]
                s[key] = X.MxMatrix(q["rows"], q["cols"], q["codes"], q["scales"])
        if op in ("quantize", "linear"):
            s["to"] = X.MxMatrix(m, k)
        if op == "backward":
            s["dy_rows"], s["dy_cols"] = X.MxMatrix(m, n), X.MxMatrix(n, m)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "adamw8":
        s["t"] += 1
        g = (s["g"].float() * s["coef"]).view(-1, BLOCK8)
        m = s["m"].view(-1, BLOCK8).float() * s["ms"][:, None]
        r = s["r"].view(-1, BLOCK8).float() * s["rs"][:, None]
        m = BETAS[0] * m + (1.0 - BETAS[0]) * g
        v = BETAS[1] * (r * r) + (1.0 - BETAS[1]) * (g * g)
        r = torch.sqrt(v)
        root = r * (1.0 / math.sqrt(1.0 - BETAS[1] ** s["t"])) + EPS
        s["p"].copy_((1.0 - RATE * DECAY) * s["p"] - RATE / (1.0 - BETAS[0] ** s["t"]) * (m / root).view(-1))
        for code, scale, x in (("m", "ms", m), ("r", "rs", r)):
            c, k = _to8(x, code == "r")
            s[code].copy_(c.view(-1))
            s[scale].copy_(k)
        out = {key: s[key] for key in ("p", "m", "ms", "r", "rs")}
        if case["copy"]:
            out["model"] = s["model"].copy_(s["p"])
        return out
    if op == "quantize":
        q, e = _round4(_padded(s["x"]))
        s["values"].copy_((q * _two(e)[:, :, None]).reshape(q.shape[0], -1)[:, :case["k"]])
        return {"values": s["values"]}
    if op == "backward":
        s["dx"].copy_(_times(_to4(s["dy"]), s["w"])[:, :case["k"]])
        s["dw"].copy_(_times(_to4(s["dy"].t()), s["x"]))
        return {"dx": s["dx"], "dw": s["dw"]}
    y = _times(s["x"] if op == "product" else _to4(s["x"]), s["w"])
    s["y"].copy_(y if s["bias"] is None else y + s["bias"])
    return {"y": s["y"]}


def _own(s):
    case, op = s["case"], s["case"]["op"]
    if op == "adamw8":
        s["t"] += 1
        s["plan"].mc_adamw8(s["t"], RATE, BETAS, EPS, DECAY, coef=s["coef"])
        out = {key: s[key] for key in ("p", "m", "ms", "r", "rs")}
        if case["copy"]:
            out["model"] = s["model"]
        return out
    if op == "quantize":
        s["mx"].mc_mx_quantize(s["x"], by_rows=s["to"], values=s["values"])
        return {"values": s["values"]}
    if op == "backward":
        s["mx"].mc_mx_quantize(s["dy"], by_rows=s["dy_rows"], by_cols=s["dy_cols"])
        s["mx"].mc_mx_matmul(s["dy_rows"], s["w"], s["dx"])
        s["mx"].mc_mx_matmul(s["dy_cols"], s["x"], s["dw"])
        return {"dx": s["dx"], "dw": s["dw"]}
    a = s["x"]
    if op == "linear":
        a = s["to"]
        s["mx"].mc_mx_quantize(s["x"], by_rows=a)
    s["mx"].mc_mx_matmul(a, s["w"], s["y"], bias=s["bias"])
    return {"y": s["y"]}


# ---- the same in 64 bits -------------------------------------------------------------------------------------------
def _power(e):
    """2^e in 64 bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest4(x):
    """Values rounded to four bits under their blocks' scales, in 64 bits, from the distances' borders."""
    x = x.double()
    rows, cols = x.shape
    filled = torch.nn.functional.pad(x, (0, -cols % BLOCK4)).reshape(rows, -1, BLOCK4)
    top = filled.abs().amax(2, keepdim=True)
    scale = _power(torch.floor(torch.log2(top.clamp(min=2.0 ** -126))) - 3)
    for _ in range(3):                                      # up to where the largest value is at most 7, whatever the logarithm's rounding
        scale = torch.where(top > 7.0 * scale, 2.0 * scale, scale)
    scale = scale.clamp(min=2.0 ** -127)
    a = filled.abs() / scale
    q = 0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75) + (a > 2.5) + (a >= 3.5) + 2.0 * (a > 5.0)
    return (q * scale * torch.sign(filled)).reshape(rows, -1)[:, :cols]


def _held4(q):
    """A quantised matrix's values in 64 bits, bit field by bit field."""
    steps = (q["cols"] + STEP_K - 1) // STEP_K
    byte = q["codes"].view(-1, steps, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(-1, steps * 64)[:q["rows"]].short()
    four = torch.stack([byte % 16, byte // 16], 2).reshape(q["rows"], -1)
    exponent, half = four % 8 // 2, (four % 2).double()
    x = torch.where(exponent == 0, 0.5 * half, _power(exponent - 1) * (1.0 + 0.5 * half))
    x = torch.where(four >= 8, -x, x)
    s = q["scales"].view(-1, steps, 4, 16, 4).permute(0, 4, 3, 1, 2).reshape(-1, steps * 4)[:q["rows"]]
    return (x.view(q["rows"], -1, BLOCK4) * _power(s.short() - 127)[:, :, None]).reshape(q["rows"], -1)[:, :q["cols"]]


def exact(case, seed):
    f64 = torch.float64
    if case["op"] == "adamw8":
        i, t = _list_inputs(case, seed), STEP + 1
        old = lambda c, s: (i[c].float().to(f64).view(-1, BLOCK8) * i[s].to(f64)[:, None]).reshape(-1)  # noqa: E731
        here = i["g"].to(f64) * i["coef"].to(f64)
        m = BETAS[0] * old("m", "ms") + (1.0 - BETAS[0]) * here
        v = BETAS[1] * old("r", "rs").square() + (1.0 - BETAS[1]) * here.square()
        p = i["p"].to(f64)
        p = p - RATE * (DECAY * p + m / (1.0 - BETAS[0] ** t) / ((v / (1.0 - BETAS[1] ** t)).sqrt() + EPS))
        out = {"p": p}
        for code, scale, x in (("m", "ms", m.view(-1, BLOCK8)), ("r", "rs", v.sqrt().view(-1, BLOCK8))):
            out[scale] = x.abs().amax(1) / TOP8
            out[code] = torch.where(out[scale][:, None] > 0, x / out[scale][:, None], 0.0).reshape(-1)       # before it is rounded
        if case["copy"]:
            out["model"] = p
        return out
    i = _matrix_inputs(case, seed)
    if case["op"] == "quantize":
        return {"values": _nearest4(i["x"])}
    if case["op"] == "backward":
        return {"dx": _nearest4(i["dy"]) @ _held4(i["w"]).t(), "dw": _nearest4(i["dy"].t()) @ _held4(i["x"]).t()}
    y = (_held4(i["x"]) if case["op"] == "product" else _nearest4(i["x"])) @ _held4(i["w"]).t()
    return {"y": y if i["bias"] is None else y + i["bias"].to(f64)}
