"""Binding of a training step in few bits (the C ABI in include/mergecomp_mx.h): AdamW with moments in 8 bits over a model's list of
tensors, microscaled 4-bit quantisation of matrices and products of such matrices.

Like step.py it marshals arguments only; tensors are checked where they are handed over.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from . import binding as B
from . import step as S

LISTS = {"grads": 0, "params": 1, "model": 2, "exp_avg": 3, "exp_avg_sq": 4, "exp_avg_scale": 5, "exp_avg_sq_scale": 6}
BLOCK8 = 128                                     # elements of a moment that share a scale
ROWS, STEP = 16, 128                             # a tile of a quantised matrix

EXPORTS = ["mc_step8_create", "mc_step8_destroy", "mc_step8_bind", "mc_adamw8", "mc_mx_code_bytes", "mc_mx_scale_bytes",
           "mc_mx_create", "mc_mx_destroy", "mc_mx_quantize", "mc_mx_matmul"]


class McMxMatrix(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64)]


class McMxSource(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("stride", C.c_int64), ("dtype", C.c_int32)]


class McMxResult(C.Structure):
    _fields_ = [("out", C.c_void_p), ("stride", C.c_int64), ("dtype", C.c_int32), ("accumulate", C.c_int32), ("bias", C.c_void_p)]


_declared = None


def lib():
    """The loaded library with these operators' signatures."""
    global _declared
    L = S.lib()
    if _declared is not L:
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.mc_step8_create.argtypes = [C.POINTER(vp), vp, i32, i32, i32, vp]
        L.mc_step8_destroy.argtypes = [vp]
        L.mc_step8_bind.argtypes = [vp, i32, vp, vp]
        L.mc_adamw8.argtypes = [vp, C.POINTER(S.McAdamwConfig), vp, vp]
        for f in (L.mc_mx_code_bytes, L.mc_mx_scale_bytes):
            f.argtypes = [i64, i64]
            f.restype = C.c_size_t
        L.mc_mx_create.argtypes = [C.POINTER(vp)]
        L.mc_mx_destroy.argtypes = [vp]
        L.mc_mx_quantize.argtypes = [vp, C.POINTER(McMxSource), C.POINTER(McMxMatrix), C.POINTER(McMxMatrix), vp, i64, vp]
        L.mc_mx_matmul.argtypes = [vp, C.POINTER(McMxMatrix), C.POINTER(McMxMatrix), C.POINTER(McMxResult), vp]
        _declared = L
    return L


class _NoFastCalls:
    """Stands for the extension module's calls where there is no module: no argument is in a form that it takes."""

    @staticmethod
    def quantize(*args):
        return None
    matmul = adamw8 = quantize


def _fast(device):
    """The extension module's calls for tensors on a device."""
    L = lib()
    try:
        return B._fastcall().MxCalls(torch.float32, torch.bfloat16, torch.float16, MxMatrix, device.index,
                                     *[C.cast(f, C.c_void_p).value for f in (L.mc_mx_quantize, L.mc_mx_matmul, L.mc_adamw8)])
    except ImportError:                          # (the library's own loading has warned)
        return _NoFastCalls()


class Step8:
    """One model's list of tensors whose moments are held in 8 bits, on the current device: wraps mc_step8.  All that is handed over later has to
    be on that device.  A graph that holds its calls is replayed only while it lives, with the numbers (step, lr, ...) that they were captured with.

    grad_dtype   type of the gradients
    model_dtype  type of the copy of the weights that the model computes with, or None for no such copy
    no_decay     per tensor, whether weight decay leaves it out
    """

    def __init__(self, numel: Sequence[int], grad_dtype="float32", model_dtype=None, no_decay: Optional[Sequence[bool]] = None):
        self.numel = [int(n) for n in numel]
        n = len(self.numel)
        if no_decay is not None and len(no_decay) != n:
            raise ValueError(f"no_decay: one entry for each of the {n} tensors")
        if model_dtype is not None and S.dtype_id(model_dtype) == S.MC_DTYPE_F32:
            raise ValueError("model_dtype: 16 bits, or None (the weights themselves are 32 bits)")
        ids = {v: k for k, v in S.DTYPE_IDS.items()}
        grad, model = S.dtype_id(grad_dtype), S.dtype_id(model_dtype)
        self.dtypes = {"grads": ids[grad], "params": torch.float32, "model": ids.get(model), "exp_avg": torch.uint8, "exp_avg_sq": torch.uint8,
                       "exp_avg_scale": torch.float32, "exp_avg_sq_scale": torch.float32}
        self._kept = {}
        self._h = C.c_void_p()
        self._at = 0                             # the same as an int
        nm = (C.c_int64 * max(n, 1))(*self.numel)
        nd = None if no_decay is None else (C.c_uint8 * max(n, 1))(*[1 if x else 0 for x in no_decay])
        B._check(lib().mc_step8_create(C.byref(self._h), nm, n, grad, model, nd), "mc_step8_create")
        self._at = self._h.value
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._fast = _fast(self._device)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().mc_step8_destroy(self._h)
            self._h = None
            self._at = 0
            self._kept = {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def moments(self) -> dict:
        """The four lists of moments of a training that begins: zeros on the handle's device, written on torch's current stream, in the form that bind() takes."""
        blocks = [(n + BLOCK8 - 1) // BLOCK8 for n in self.numel]
        return {name: [torch.zeros(n, dtype=self.dtypes[name], device=self._device) for n in (blocks if name.endswith("scale") else self.numel)]
                for name in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")}

    def bind(self, stream=None, **lists) -> None:
        """Hands over lists of tensors (any iterables), one tensor for each of the model: grads, params, model; exp_avg and exp_avg_sq (bytes, as many as
        elements), exp_avg_scale and exp_avg_sq_scale (floats, one for 128 elements).  A list holds until it is handed over again; its
        tensors are kept alive until then."""
        lists = {name: list(tensors) for name, tensors in lists.items()}         # gone through once: it may be a generator
        for name, tensors in lists.items():
            if name not in LISTS:
                raise ValueError(f"{name}: one of {', '.join(LISTS)}")
            kind = self.dtypes[name]
            if kind is None:
                raise ValueError("model: the handle was made without a model_dtype")
            if len(tensors) != len(self.numel):
                raise ValueError(f"{name}: {len(self.numel)} tensors, not {len(tensors)}")
            for i, (t, n) in enumerate(zip(tensors, self.numel)):
                count = (n + BLOCK8 - 1) // BLOCK8 if name.endswith("scale") else n
                if t.numel() != count or not t.is_contiguous() or t.device != self._device or t.dtype is not kind:
                    raise ValueError(f"{name}[{i}]: {count} contiguous values of {kind} on {self._device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        handle = S._stream_on(stream, self._device)
        for name, tensors in lists.items():
            B._check(lib().mc_step8_bind(self._h, LISTS[name], B.ptr_array(tensors), handle), "mc_step8_bind")
            self._kept[name] = tensors

    def mc_adamw8(self, step: int, lr: float, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                  coef=None, stream=None) -> None:
        """coef: one float on the device that the gradients are multiplied by, such as the second of mc_grad_norm.

        Roots of second moments that become smaller are followed up to betas[1] of about 0.98.  With the default, AdamW's own, they stay where they were, several times
        too large, and updates too small: what rounds to the same 8-bit code every time never adds up (the header has figures)."""
        rc = self._fast.adamw8(self._at, step, lr, betas[0], betas[1], eps, weight_decay, coef, B._raw_stream) if stream is None else None
        if rc is None:
            cfg = S.McAdamwConfig(lr, betas[0], betas[1], eps, weight_decay, step)
            rc = lib().mc_adamw8(self._h, C.byref(cfg), None if coef is None else S._vector(coef, "coef", 1, self._device), S._stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_adamw8")


class MxMatrix:
    """rows x cols values in microscaled 4-bit floating point: the two buffers of mc_mx_matrix, made here (zeros on the current device, written on torch's current
    stream, which calls on another one have to wait for) or handed over (bytes, contiguous, on one device, mc_mx_code_bytes and mc_mx_scale_bytes of them).  A matrix keeps its buffers: another one's are another matrix."""

    rows = property(lambda self: self._rows)
    cols = property(lambda self: self._cols)
    codes = property(lambda self: self._codes)
    scales = property(lambda self: self._scales)

    def __init__(self, rows: int, cols: int, codes=None, scales=None):
        self._rows, self._cols = int(rows), int(cols)
        if self.rows < 0 or self.cols < 1 or max(self.rows, self.cols) >= 2 ** 31 - 2 ** 16:
            raise ValueError(f"{rows} x {cols}: rows from 0 and columns from 1 on, below 2^31 - 2^16")
        if (codes is None) != (scales is None):
            raise ValueError("codes and scales: both or neither")
        sizes = lib().mc_mx_code_bytes(self.rows, self.cols), lib().mc_mx_scale_bytes(self.rows, self.cols)
        if codes is None:
            device = torch.device("cuda", torch.cuda.current_device())
            codes, scales = (torch.zeros(n, dtype=torch.uint8, device=device) for n in sizes)
        for name, t, n in (("codes", codes, sizes[0]), ("scales", scales, sizes[1])):
            if t.dtype is not torch.uint8 or t.numel() != n or not t.is_contiguous() or t.device != codes.device or not t.is_cuda:
                raise ValueError(f"{name}: {n} contiguous bytes on one device, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        self._codes, self._scales = codes, scales
        self._c = McMxMatrix(codes.data_ptr(), scales.data_ptr(), self.rows, self.cols)
        self._at = C.addressof(self._c)
        self._device, self._index = codes.device, codes.device.index


def _matrix(m, name: str, device, rows=None, cols=None):
    if not isinstance(m, MxMatrix) or m._device != device or (rows is not None and m.rows != rows) or (cols is not None and m.cols != cols):
        what = "an MxMatrix" if rows is None or cols is None else f"an MxMatrix of {rows} x {cols}"
        raise ValueError(f"{name}: {what} on {device}, not {f'{m.rows} x {m.cols} on {m._device}' if isinstance(m, MxMatrix) else type(m).__name__}")
    return C.byref(m._c)


class Mx:
    """Scratch of the calls over quantised matrices, on the current device, where their tensors have to be: wraps mc_mx.  A graph that holds its calls is replayed only
    while it lives."""

    def __init__(self):
        self._h = C.c_void_p()
        self._at = 0                             # the same as an int
        B._check(lib().mc_mx_create(C.byref(self._h)), "mc_mx_create")
        self._at = self._h.value
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._fast = _fast(self._device)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().mc_mx_destroy(self._h)
            self._h = None
            self._at = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def mc_mx_quantize(self, x, by_rows=None, by_cols=None, values=None, stream=None) -> None:
        """x: rows of contiguous values.  by_rows: an MxMatrix of x's shape; by_cols: one of the transposed shape; values: of x's shape and type (it may be
        x), what by_rows stands for."""
        rc = self._fast.quantize(self._at, x, by_rows, by_cols, values, B._raw_stream) if stream is None else None
        if rc is None:
            rc = self._quantize(x, by_rows, by_cols, values, S._stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_mx_quantize")

    def _quantize(self, x, by_rows, by_cols, values, stream) -> int:
        """The same through ctypes, which says what is wrong with an argument."""
        rows, cols, stride = S._rows(x, "x", self._device)
        at, vstride = None, 0
        if values is not None:
            vrows, vcols, vstride = S._rows(values, "values", self._device)
            if vrows != rows or vcols != cols or values.dtype is not x.dtype:
                raise ValueError(f"values: x's shape and type, not {tuple(values.shape)} of {values.dtype}")
            at = values.data_ptr()
        src = McMxSource(x.data_ptr(), rows, cols, stride, S.DTYPE_IDS[x.dtype])
        r = None if by_rows is None else _matrix(by_rows, "by_rows", self._device, rows, cols)
        c = None if by_cols is None else _matrix(by_cols, "by_cols", self._device, cols, rows)
        return lib().mc_mx_quantize(self._h, C.byref(src), r, c, at, vstride, stream)

    def mc_mx_matmul(self, a, b, out, bias=None, accumulate: bool = False, stream=None) -> None:
        """out = a b^T (+ bias, b.rows floats) (+ out as it was), out: a.rows rows of b.rows contiguous values."""
        rc = self._fast.matmul(self._at, a, b, out, bias, accumulate, B._raw_stream) if stream is None else None
        if rc is None:
            rc = self._matmul(a, b, out, bias, accumulate, S._stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_mx_matmul")

    def _matmul(self, a, b, out, bias, accumulate, stream) -> int:
        """The same through ctypes, which says what is wrong with an argument."""
        pa, pb = _matrix(a, "a", self._device), _matrix(b, "b", self._device)
        rows, cols, stride = S._rows(out, "out", self._device)
        if rows != a.rows or cols != b.rows or a.cols != b.cols:
            raise ValueError(f"out: {a.rows} x {b.rows} of sums over {a.cols} and {b.cols} columns, not {rows} x {cols}")
        y = McMxResult(out.data_ptr(), stride, S.DTYPE_IDS[out.dtype], 1 if accumulate else 0, None if bias is None else S._vector(bias, "bias", cols, self._device))
        return lib().mc_mx_matmul(self._h, pa, pb, C.byref(y), stream)
