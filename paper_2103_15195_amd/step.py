"""Binding of the operators around a step's exchange of gradients (the C ABI in include/mergecomp_step.h): the global
gradient norm, clipping and AdamW over a model's list of tensors, token log-probabilities and the clipped policy loss
over rows of logits.

Like binding.py it marshals arguments only, tensors are passed by ``data_ptr()`` and ``stream=None`` is torch's current
stream.  Tensors are checked where they are handed over, since the kernels go by sizes that are fixed then.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from . import binding as B

MC_DTYPE_NONE, MC_DTYPE_F32, MC_DTYPE_BF16, MC_DTYPE_F16 = -1, 0, 1, 2
DTYPE_IDS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
LISTS = {"grads": 0, "clipped": 1, "params": 2, "exp_avg": 3, "exp_avg_sq": 4, "model": 5}

EXPORTS = ["mc_step_create", "mc_step_destroy", "mc_step_bind", "mc_grad_norm", "mc_grad_clip", "mc_adamw",
           "mc_loss_create", "mc_loss_destroy", "mc_token_logp", "mc_policy_loss"]


class McAdamwConfig(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("step", C.c_int64)]


class McLogits(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("labels", C.c_void_p), ("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64),
                ("dtype", C.c_int32), ("temperature", C.c_float)]


class McPolicy(C.Structure):
    _fields_ = [("old_logp", C.c_void_p), ("advantages", C.c_void_p), ("weights", C.c_void_p), ("ref_logp", C.c_void_p),
                ("clip_low", C.c_float), ("clip_high", C.c_float), ("kl_coef", C.c_float), ("grad_scale", C.c_float),
                ("sums", C.c_void_p), ("logp", C.c_void_p), ("dlogits", C.c_void_p), ("dlogits_stride", C.c_int64)]


_declared = None


def lib():
    """The loaded library with these operators' signatures."""
    global _declared
    L = B.lib()
    if _declared is not L:
        vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
        L.mc_step_create.argtypes = [C.POINTER(vp), vp, i32, i32, i32, vp]
        L.mc_step_destroy.argtypes = [vp]
        L.mc_step_bind.argtypes = [vp, i32, vp, vp]
        L.mc_grad_norm.argtypes = [vp, f32, f32, vp, vp]
        L.mc_grad_clip.argtypes = [vp, f32, f32, vp, vp]
        L.mc_adamw.argtypes = [vp, C.POINTER(McAdamwConfig), vp, vp]
        L.mc_loss_create.argtypes = [C.POINTER(vp)]
        L.mc_loss_destroy.argtypes = [vp]
        L.mc_token_logp.argtypes = [vp, C.POINTER(McLogits), vp, vp]
        L.mc_policy_loss.argtypes = [vp, C.POINTER(McLogits), C.POINTER(McPolicy), vp]
        try:
            L.fast_step = B._fastcall().StepCalls(torch.float32, torch.bfloat16, torch.float16, torch.int64, *[C.cast(f, vp).value for f in (
                L.mc_token_logp, L.mc_policy_loss, L.mc_grad_norm, L.mc_grad_clip, L.mc_adamw)])
        except ImportError:                      # (the library's own loading has warned)
            L.fast_step = _NoFastCalls()
        _declared = L
    return L


class _NoFastCalls:
    """Stands for the extension module's calls where there is no module: no argument is in a form that it takes."""

    @staticmethod
    def token_logp(*args):
        return None
    policy_loss = grad_norm = grad_clip = adamw = token_logp

    def on(self, device):
        return self


def dtype_id(dtype) -> int:
    """mc_dtype of a torch dtype or its name; None: no type."""
    if dtype is None:
        return MC_DTYPE_NONE
    kind = getattr(torch, dtype, dtype) if isinstance(dtype, str) else dtype
    if kind not in DTYPE_IDS:
        raise ValueError(f"{dtype}: one of {', '.join(map(str, DTYPE_IDS))}")
    return DTYPE_IDS[kind]


_F32, _I64 = torch.float32, torch.int64


def _vector(tensor, name: str, count: int, device, kind=_F32) -> int:
    """The address of a contiguous tensor of `count` elements on the handle's device."""
    if tensor.dtype is not kind or tensor.numel() != count or tensor.device != device or not tensor.is_contiguous():
        raise ValueError(f"{name}: {count} contiguous values of {kind} on {device}, not {tuple(tensor.shape)} of {tensor.dtype} on {tensor.device}")
    return tensor.data_ptr()


def _rows(x, name: str, device=None):
    """(rows, columns, elements from row to row) of a two-dimensional tensor whose rows are contiguous, on the handle's device (None: on any)."""
    shape, step = x.shape, x.stride()
    if len(shape) != 2 or not (x.is_cuda if device is None else x.device == device) or x.dtype not in DTYPE_IDS or (step[1] != 1 and shape[1] > 1):
        raise ValueError(f"{name}: rows of contiguous values on {device or 'the device'}, of {', '.join(map(str, DTYPE_IDS))}, not {tuple(shape)} of {x.dtype} on {x.device}")
    return shape[0], shape[1], step[0] if shape[0] > 1 else max(step[0], shape[1])


def _stream_on(stream, device) -> Optional[int]:
    """The stream's handle; None: torch's current stream, for which the handle's device has to be the current one."""
    at = torch.device("cuda", torch.cuda.current_device()) if stream is None else stream.device if hasattr(stream, "cuda_stream") else device
    if at != device:
        raise ValueError(f"{'the current device' if stream is None else 'stream'}: {at}, but the handle was made on {device}")
    return B._stream_handle(stream)


class Step:
    """One model's list of tensors on the current device: wraps mc_step.  All that is handed over later has to be on that device.

    grad_dtype   type of the gradients (and of what mc_grad_clip writes)
    model_dtype  type of the copy of the weights that the model computes with, or None for no such copy
    no_decay     per tensor, whether weight decay leaves it out
    """

    def __init__(self, numel: Sequence[int], grad_dtype="float32", model_dtype=None, no_decay: Optional[Sequence[bool]] = None):
        self.numel = [int(n) for n in numel]
        n = len(self.numel)
        if no_decay is not None and len(no_decay) != n:
            raise ValueError(f"no_decay: one entry for each of the {n} tensors")
        if model_dtype is not None and dtype_id(model_dtype) == MC_DTYPE_F32:
            raise ValueError("model_dtype: 16 bits, or None (the weights themselves are 32 bits)")
        self.dtypes = {"grads": dtype_id(grad_dtype), "clipped": dtype_id(grad_dtype), "model": dtype_id(model_dtype),
                       "params": MC_DTYPE_F32, "exp_avg": MC_DTYPE_F32, "exp_avg_sq": MC_DTYPE_F32}
        self._kept = {}
        self._h = C.c_void_p()
        self._at = 0                             # the same as an int
        nm = (C.c_int64 * max(n, 1))(*self.numel)
        nd = None if no_decay is None else (C.c_uint8 * max(n, 1))(*[1 if x else 0 for x in no_decay])
        B._check(lib().mc_step_create(C.byref(self._h), nm, n, self.dtypes["grads"], self.dtypes["model"], nd), "mc_step_create")
        self._at = self._h.value
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._fast = lib().fast_step.on(self._device.index)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().mc_step_destroy(self._h)
            self._h = None
            self._at = 0
            self._kept = {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def bind(self, stream=None, **lists) -> None:
        """Hands over lists of tensors (any iterables), one tensor for each of the model: grads, clipped, params, exp_avg, exp_avg_sq, model.
        A list holds until it is handed over again; its tensors are kept alive until then."""
        lists = {name: list(tensors) for name, tensors in lists.items()}         # gone through once: it may be a generator
        for name, tensors in lists.items():
            if name not in LISTS:
                raise ValueError(f"{name}: one of {', '.join(LISTS)}")
            if name == "model" and self.dtypes["model"] == MC_DTYPE_NONE:
                raise ValueError("model: the handle was made without a model_dtype")
            if len(tensors) != len(self.numel):
                raise ValueError(f"{name}: {len(self.numel)} tensors, not {len(tensors)}")
            for i, (t, n) in enumerate(zip(tensors, self.numel)):
                if t.numel() != n or not t.is_contiguous() or t.device != self._device or DTYPE_IDS.get(t.dtype) != self.dtypes[name]:
                    raise ValueError(f"{name}[{i}]: {n} contiguous elements of the list's type on {self._device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        handle = _stream_on(stream, self._device)
        for name, tensors in lists.items():
            B._check(lib().mc_step_bind(self._h, LISTS[name], B.ptr_array(tensors), handle), "mc_step_bind")
            self._kept[name] = tensors

    def mc_grad_norm(self, max_norm: float, out, scale: float = 1.0, stream=None) -> None:
        """out: two floats on the device, the norm of scale * gradients and the coefficient that clips them to max_norm."""
        rc = self._fast.grad_norm(self._at, scale, max_norm, out, B._raw_stream) if stream is None else None
        if rc is None:
            rc = lib().mc_grad_norm(self._h, scale, max_norm, _vector(out, "out", 2, self._device), _stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_grad_norm")

    def mc_grad_clip(self, max_norm: float, out, scale: float = 1.0, stream=None) -> None:
        """mc_grad_norm, and the gradients times the coefficient into the list `clipped`, or in place where it is not bound."""
        rc = self._fast.grad_clip(self._at, scale, max_norm, out, B._raw_stream) if stream is None else None
        if rc is None:
            rc = lib().mc_grad_clip(self._h, scale, max_norm, _vector(out, "out", 2, self._device), _stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_grad_clip")

    def mc_adamw(self, step: int, lr: float, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                 coef=None, stream=None) -> None:
        """coef: one float on the device that the gradients are multiplied by, such as the second of mc_grad_norm."""
        rc = self._fast.adamw(self._at, step, lr, betas[0], betas[1], eps, weight_decay, coef, B._raw_stream) if stream is None else None
        if rc is None:
            cfg = McAdamwConfig(lr, betas[0], betas[1], eps, weight_decay, step)
            rc = lib().mc_adamw(self._h, C.byref(cfg), None if coef is None else _vector(coef, "coef", 1, self._device), _stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_adamw")


class PolicyLoss:
    """Scratch of the calls over rows of logits, on the current device, where their tensors have to be: wraps mc_loss."""

    def __init__(self):
        self._h = C.c_void_p()
        self._at = 0                             # the same as an int
        B._check(lib().mc_loss_create(C.byref(self._h)), "mc_loss_create")
        self._at = self._h.value
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._fast = lib().fast_step.on(self._device.index)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().mc_loss_destroy(self._h)
            self._h = None
            self._at = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def mc_token_logp(self, logits, labels, logp, temperature: float = 1.0, stream=None) -> None:
        """logp[r] = log-probability of labels[r] under logits[r] / temperature; 0 where the label is none of the row's."""
        rc = self._fast.token_logp(self._at, logits, labels, logp, temperature, B._raw_stream) if stream is None else None
        if rc is None:
            rows, vocab, stride = _rows(logits, "logits", self._device)
            x = McLogits(logits.data_ptr(), _vector(labels, "labels", rows, self._device, _I64), rows, vocab, stride, DTYPE_IDS[logits.dtype], temperature)
            rc = lib().mc_token_logp(self._h, C.byref(x), _vector(logp, "logp", rows, self._device), _stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_token_logp")

    def mc_policy_loss(self, logits, labels, old_logp, advantages, *, sums, weights=None, ref_logp=None, clip: Tuple[float, float] = (0.2, 0.2),
                       kl_coef: float = 0.0, temperature: float = 1.0, grad_scale: float = 1.0, logp=None, dlogits=None, stream=None) -> None:
        """The loss of mergecomp_step.h and, in dlogits (which may be the logits), grad_scale times its gradient.
        sums: 8 floats on the device: loss, policy term, KL term, clipped weight, weight; as int32 rows that took part, rows
        whose label is none of the row's; 0."""
        rc = self._fast.policy_loss(self._at, logits, labels, old_logp, advantages, weights, ref_logp, clip[0], clip[1], kl_coef, temperature,
                                    grad_scale, sums, logp, dlogits, B._raw_stream) if stream is None else None
        if rc is None:
            rc = self._policy_loss(logits, labels, old_logp, advantages, sums, weights, ref_logp, clip, kl_coef, temperature, grad_scale, logp,
                                   dlogits, _stream_on(stream, self._device))
        if rc:
            raise B.McError(rc, "mc_policy_loss")

    def _policy_loss(self, logits, labels, old_logp, advantages, sums, weights, ref_logp, clip, kl_coef, temperature, grad_scale, logp, dlogits, stream) -> int:
        """The same through ctypes, which says what is wrong with an argument."""
        rows, vocab, stride = _rows(logits, "logits", self._device)
        x = McLogits(logits.data_ptr(), _vector(labels, "labels", rows, self._device, _I64), rows, vocab, stride, DTYPE_IDS[logits.dtype], temperature)
        slopes, dstride = None, 0
        if dlogits is not None:
            drows, dvocab, dstride = _rows(dlogits, "dlogits", self._device)
            if drows != rows or dvocab != vocab or dlogits.dtype is not logits.dtype:
                raise ValueError(f"dlogits: the logits' shape and type, not {tuple(dlogits.shape)} of {dlogits.dtype}")
            slopes = dlogits.data_ptr()
        p = McPolicy(_vector(old_logp, "old_logp", rows, self._device), _vector(advantages, "advantages", rows, self._device),
                     None if weights is None else _vector(weights, "weights", rows, self._device), None if ref_logp is None else _vector(ref_logp, "ref_logp", rows, self._device),
                     clip[0], clip[1], kl_coef, grad_scale, _vector(sums, "sums", 8, self._device), None if logp is None else _vector(logp, "logp", rows, self._device), slopes, dstride)
        return lib().mc_policy_loss(self._h, C.byref(x), C.byref(p), stream)
