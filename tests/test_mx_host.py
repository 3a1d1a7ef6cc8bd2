"""The binding of the operators in mergecomp_mx.h without a device: what the header declares is there, and what a tensor, a matrix, a stream or the current
device has to be is looked at before the library is called, by either route.  Stand-ins for device tensors and a recorder in the library's place."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import mx as X
from paper_2103_15195_amd import step as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
vp, i32 = C.c_void_p, C.c_int32


def test_header_exports_and_structures():
    text = open(os.path.join(ROOT, "include", "mergecomp_mx.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(mc_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(X.EXPORTS)
    L = X.lib()
    assert all(hasattr(L, n) for n in names)
    assert (C.sizeof(X.McMxMatrix), C.sizeof(X.McMxSource), C.sizeof(X.McMxResult)) == (32, 40, 32)
    assert [int(n) for n in re.findall(r"MC_LIST8_\w+ = (\d)", text)] == list(X.LISTS.values())


class Tensor:
    """Stands for a tensor on cuda:`at`, or in host memory (-1)."""
    def __init__(self, shape, dtype=torch.float32, at=1, address=4096, strides=None):
        self.shape, self.dtype, self.is_cuda, self.address = tuple(shape), dtype, at >= 0, address
        self.device = torch.device("cuda", at) if at >= 0 else torch.device("cpu")
        self.strides = strides or tuple(torch.empty(shape, device="meta").stride())

    def stride(self):
        return self.strides

    def numel(self):
        return torch.Size(self.shape).numel()

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def data_ptr(self):
        return self.address


class Stream:
    def __init__(self, at):
        self.device, self.cuda_stream = torch.device("cuda", at), 0x7000 + at


def matrix(rows, cols, at=1):
    steps = -(-cols // 128)
    return X.MxMatrix(rows, cols, Tensor((-(-rows // 16) * steps * 1024,), torch.uint8, at, 1 << 20), Tensor((-(-rows // 64) * steps * 256,), torch.uint8, at, 1 << 21))


def fields(p, kind):
    if not p:
        return None
    s = C.cast(p, C.POINTER(kind))[0]
    return {name: getattr(s, name) for name, _ in kind._fields_}


@pytest.fixture(params=["module", "ctypes"])
def seen(request, monkeypatch):
    """Handles on cuda:1, which is the current device, and what arrives at the library."""
    calls = []
    def quantize(h, src, r, c, v, vs, st):
        calls.append(("quantize", fields(src, X.McMxSource), fields(r, X.McMxMatrix), fields(c, X.McMxMatrix), v, vs, st))
        return 0
    def matmul(h, a, b, y, st):
        calls.append(("matmul", fields(a, X.McMxMatrix), fields(b, X.McMxMatrix), fields(y, X.McMxResult), st))
        return 0
    def adamw8(h, cfg, coef, st):
        calls.append(("adamw8", fields(cfg, S.McAdamwConfig), coef, st))
        return 0
    keep = [C.CFUNCTYPE(i32, vp, vp, vp, vp, vp, C.c_int64, vp)(quantize), C.CFUNCTYPE(i32, vp, vp, vp, vp, vp)(matmul), C.CFUNCTYPE(i32, vp, vp, vp, vp)(adamw8)]

    class Library:
        mc_mx_quantize, mc_mx_matmul, mc_adamw8 = keep
        mc_step8_bind = staticmethod(lambda *a: calls.append(("bind", a[1])) or 0)
        mc_mx_code_bytes, mc_mx_scale_bytes = X.lib().mc_mx_code_bytes, X.lib().mc_mx_scale_bytes
    monkeypatch.setattr(X, "lib", lambda: Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(B, "_raw_stream", B._fastcall().RawStream(lambda d: 0x7000 + d, lambda: 1))
    fast = X._fast(torch.device("cuda", 1)) if request.param == "module" else X._NoFastCalls()
    mx, step = X.Mx.__new__(X.Mx), X.Step8.__new__(X.Step8)
    for h in (mx, step):
        h._h, h._at, h._device, h._fast = None, 8, torch.device("cuda", 1), fast
    step.numel, step._kept = [200], {}
    step.dtypes = {"grads": torch.bfloat16, "params": torch.float32, "model": None, "exp_avg": torch.uint8, "exp_avg_sq": torch.uint8, "exp_avg_scale": torch.float32, "exp_avg_sq_scale": torch.float32}
    return calls, mx, step, keep


def test_arguments_arrive(seen):
    calls, mx, step, _ = seen
    r, c, x = matrix(20, 300), matrix(300, 20), Tensor((20, 300), torch.bfloat16, strides=(310, 1))
    v = Tensor((20, 300), torch.bfloat16, address=8192)
    mx.mc_mx_quantize(x, by_rows=r, by_cols=c, values=v)
    at = lambda m: dict(codes=1 << 20, scales=1 << 21, rows=m.rows, cols=m.cols)  # noqa: E731
    assert calls.pop() == ("quantize", dict(data=4096, rows=20, cols=300, stride=310, dtype=1), at(r), at(c), 8192, 300, 0x7001)
    mx.mc_mx_quantize(x, by_cols=c)
    assert calls.pop()[2:6] == (None, at(c), None, 0)
    b, out, bias = matrix(30, 300), Tensor((20, 30), torch.float16), Tensor((30,), address=512)
    mx.mc_mx_matmul(r, b, out, bias=bias, accumulate=True)
    assert calls.pop() == ("matmul", at(r), at(b), dict(out=4096, stride=30, dtype=2, accumulate=1, bias=512), 0x7001)
    mx.mc_mx_matmul(r, b, out, stream=Stream(1))
    assert calls.pop()[3:] == (dict(out=4096, stride=30, dtype=2, accumulate=0, bias=None), 0x7001)
    step.mc_adamw8(3, 0.5, (0.25, 0.75), 1e-3, 0.125, coef=Tensor((1,), address=16))
    assert calls.pop() == ("adamw8", dict(lr=0.5, beta1=0.25, beta2=0.75, eps=1e-3, weight_decay=0.125, step=3), 16, 0x7001)
    step.mc_adamw8(step=1, lr=0.5)
    assert calls.pop()[2:] == (None, 0x7001)
    step.bind(grads=(Tensor((200,), torch.bfloat16) for _ in range(1)), exp_avg_scale=[Tensor((2,))])
    assert [calls.pop(), calls.pop()] == [("bind", 5), ("bind", 0)]


def test_what_lies_elsewhere_or_is_of_another_size(seen, monkeypatch):
    calls, mx, step, _ = seen
    r, b, x, out = matrix(20, 300), matrix(30, 300), Tensor((20, 300)), Tensor((20, 30))
    bad = [lambda: mx.mc_mx_quantize(Tensor((20, 300), at=0), by_rows=r), lambda: mx.mc_mx_quantize(Tensor((20, 300), at=-1), by_rows=r),
           lambda: mx.mc_mx_quantize(x, by_rows=matrix(20, 300, at=0)), lambda: mx.mc_mx_quantize(x, by_rows=b), lambda: mx.mc_mx_quantize(x, by_cols=r),
           lambda: mx.mc_mx_quantize(x, by_rows=x), lambda: mx.mc_mx_quantize(x, by_rows=r, values=Tensor((20, 300), torch.bfloat16)),
           lambda: mx.mc_mx_quantize(x, by_rows=r, values=Tensor((20, 300), at=0)), lambda: mx.mc_mx_quantize(x, by_rows=r, values=Tensor((20, 299))),
           lambda: mx.mc_mx_quantize(Tensor((20, 300), strides=(1, 20)), by_rows=r), lambda: mx.mc_mx_quantize(x, by_rows=r, stream=Stream(0)),
           lambda: mx.mc_mx_matmul(r, b, Tensor((20, 30), at=0)), lambda: mx.mc_mx_matmul(matrix(20, 300, at=0), b, out), lambda: mx.mc_mx_matmul(r, matrix(30, 299), out),
           lambda: mx.mc_mx_matmul(r, b, Tensor((20, 31))), lambda: mx.mc_mx_matmul(b, r, out), lambda: mx.mc_mx_matmul(r, b, out, bias=Tensor((29,))),
           lambda: mx.mc_mx_matmul(r, b, out, bias=Tensor((30,), torch.float16)), lambda: mx.mc_mx_matmul(r, b, out, bias=Tensor((30,), at=0)),
           lambda: mx.mc_mx_matmul(r, x, out), lambda: mx.mc_mx_matmul(r, b, Tensor((20, 30), torch.float64)),
           lambda: step.mc_adamw8(1, 0.5, coef=Tensor((1,), at=0)), lambda: step.mc_adamw8(1, 0.5, coef=Tensor((2,))), lambda: step.mc_adamw8(1, 0.5, stream=Stream(0)),
           lambda: step.bind(grads=[Tensor((200,))]), lambda: step.bind(exp_avg=[Tensor((200,), torch.uint8, at=0)]), lambda: step.bind(exp_avg_scale=[Tensor((3,))]),
           lambda: step.bind(model=[Tensor((200,), torch.bfloat16)]), lambda: step.bind(moments=[]), lambda: step.bind(params=[])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)                # another device is current
    monkeypatch.setattr(B, "_raw_stream", B._fastcall().RawStream(lambda d: 0x7000 + d, lambda: 0))
    for call in (lambda: mx.mc_mx_quantize(x, by_rows=r), lambda: mx.mc_mx_matmul(r, b, out), lambda: step.mc_adamw8(1, 0.5)):
        with pytest.raises(ValueError):
            call()
    assert calls == []


def test_matrices():
    for rows, cols in ((-1, 5), (5, 0), (2 ** 31, 5), (5, 2 ** 31 - 2 ** 16)):
        with pytest.raises(ValueError):
            X.MxMatrix(rows, cols, Tensor((0,), torch.uint8), Tensor((0,), torch.uint8))
    good = Tensor((2048,), torch.uint8), Tensor((256,), torch.uint8)
    m = X.MxMatrix(20, 100, *good)
    assert (m.rows, m.cols, m.codes, m.scales) == (20, 100, *good)
    for name in ("rows", "cols", "codes", "scales"):          # the library has their addresses
        with pytest.raises(AttributeError):
            setattr(m, name, None)
    for codes, scales in ((good[0], None), (None, good[1]), (good[1], good[0]), (good[0], Tensor((256,), torch.uint8, at=0)), (Tensor((2048,), torch.uint8, at=-1), good[1]),
                          (good[0], Tensor((256,), torch.int8))):
        with pytest.raises(ValueError):
            X.MxMatrix(20, 100, codes, scales)
