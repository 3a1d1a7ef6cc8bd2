"""Tensors, streams and the current device against the device that a handle was made on: what lies elsewhere is refused before the library is called.
Stand-ins for device tensors and a recorder in the library's place; needs no device."""
import ctypes as C

import pytest
import torch

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S

vp, i32 = C.c_void_p, C.c_int32
ROWS, VOCAB = 5, 11


class Tensor:
    """Stands for a tensor on cuda:`at`, or in host memory (-1)."""
    def __init__(self, shape, dtype=torch.float32, at=1, address=4096):
        self.shape, self.dtype, self.is_cuda, self.address = tuple(shape), dtype, at >= 0, address
        self.device = torch.device("cuda", at) if at >= 0 else torch.device("cpu")
        self.strides = tuple(torch.empty(shape, device="meta").stride())

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


class Recorder:
    """Stands for the library: notes the calls."""

    def __init__(self):
        self.calls = []
        for name in ("mc_step_bind", "mc_grad_norm", "mc_grad_clip", "mc_adamw", "mc_token_logp", "mc_policy_loss"):
            setattr(self, name, lambda *a, name=name: self.calls.append((name, a)) or B.MC_OK)


def handles(fast, index):
    """The Python side of a handle of each kind, made on cuda:`index`."""
    step, loss = S.Step.__new__(S.Step), S.PolicyLoss.__new__(S.PolicyLoss)
    step.numel, step.dtypes, step._kept = [3], {name: 0 for name in S.LISTS}, {}
    for h in (step, loss):
        h._h, h._at, h._device, h._fast = None, 8, torch.device("cuda", index), fast.on(index)
    return step, loss


def current(monkeypatch, index):
    """cuda:`index` is the current device."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: index)
    monkeypatch.setattr(B, "_raw_stream", B._fastcall().RawStream(lambda d: 0x7000 + d, lambda: index))


@pytest.fixture
def seen(monkeypatch):
    """What arrives, through either route."""
    r = Recorder()
    monkeypatch.setattr(S, "lib", lambda: r)
    current(monkeypatch, 1)
    keep = [C.CFUNCTYPE(i32, vp, C.POINTER(S.McLogits), vp, vp)(lambda *a: r.calls.append(("mc_token_logp", a)) or 0),
            C.CFUNCTYPE(i32, vp, C.POINTER(S.McLogits), C.POINTER(S.McPolicy), vp)(lambda *a: r.calls.append(("mc_policy_loss", a)) or 0)]
    norm = C.CFUNCTYPE(i32, vp, C.c_float, C.c_float, vp, vp)
    keep += [norm(lambda *a: r.calls.append(("mc_grad_norm", a)) or 0), norm(lambda *a: r.calls.append(("mc_grad_clip", a)) or 0),
             C.CFUNCTYPE(i32, vp, C.POINTER(S.McAdamwConfig), vp, vp)(lambda *a: r.calls.append(("mc_adamw", a)) or 0)]
    r.keep = keep
    r.fast = B._fastcall().StepCalls(torch.float32, torch.bfloat16, torch.float16, torch.int64, *[C.cast(k, vp).value for k in keep])
    return r


ROUTES = {"module": lambda seen: seen.fast, "ctypes": lambda seen: S._NoFastCalls()}


def policy_args(**other):
    a = dict(logits=Tensor((ROWS, VOCAB)), labels=Tensor((ROWS,), torch.int64), old_logp=Tensor((ROWS,)), advantages=Tensor((ROWS,)), sums=Tensor((8,)),
             weights=Tensor((ROWS,)), ref_logp=Tensor((ROWS,)), logp=Tensor((ROWS,)), dlogits=Tensor((ROWS, VOCAB)))
    return {**a, **other}


@pytest.mark.parametrize("at", [0, 2, -1])
@pytest.mark.parametrize("route", list(ROUTES))
def test_tensors_of_another_device_are_refused(seen, route, at):
    step, loss = handles(ROUTES[route](seen), 1)
    loss.mc_policy_loss(**policy_args())
    loss.mc_token_logp(Tensor((ROWS, VOCAB)), Tensor((ROWS,), torch.int64), Tensor((ROWS,)))
    step.mc_grad_norm(1.0, Tensor((2,)))
    step.mc_grad_clip(1.0, Tensor((2,)))
    step.mc_adamw(1, 1e-3, coef=Tensor((1,)))
    step.bind(grads=[Tensor((3,))])
    good = ["mc_policy_loss", "mc_token_logp", "mc_grad_norm", "mc_grad_clip", "mc_adamw", "mc_step_bind"]
    assert [name for name, _ in seen.calls] == good
    for name, tensor in policy_args().items():
        away = Tensor(tensor.shape, tensor.dtype, at)
        with pytest.raises(ValueError, match=name):
            loss.mc_policy_loss(**policy_args(**{name: away}))
        if name in ("logits", "labels", "logp"):
            with pytest.raises(ValueError, match=name):
                loss.mc_token_logp(*[away if name == n else t for n, t in policy_args().items() if n in ("logits", "labels", "logp")])
    for call in (lambda: step.mc_grad_norm(1.0, Tensor((2,), at=at)), lambda: step.mc_grad_clip(1.0, Tensor((2,), at=at)),
                 lambda: step.mc_adamw(1, 1e-3, coef=Tensor((1,), at=at)), lambda: step.bind(grads=[Tensor((3,), at=at)])):
        with pytest.raises(ValueError, match="cuda:1"):
            call()
    assert len(seen.calls) == len(good)


@pytest.mark.parametrize("route", list(ROUTES))
def test_another_current_device_is_refused(seen, route, monkeypatch):
    """Without a stream the call would go to the current device's."""
    step, loss = handles(ROUTES[route](seen), 1)
    calls = [lambda **k: loss.mc_policy_loss(**policy_args(), **k), lambda **k: loss.mc_token_logp(Tensor((ROWS, VOCAB)), Tensor((ROWS,), torch.int64), Tensor((ROWS,)), **k),
             lambda **k: step.mc_grad_norm(1.0, Tensor((2,)), **k), lambda **k: step.mc_grad_clip(1.0, Tensor((2,)), **k),
             lambda **k: step.mc_adamw(1, 1e-3, **k), lambda **k: step.bind(grads=[Tensor((3,))], **k)]
    current(monkeypatch, 0)
    for call in calls:
        with pytest.raises(ValueError, match="cuda:1"):
            call()
        with pytest.raises(ValueError, match="cuda:1"):
            call(stream=Stream(0))
    assert not seen.calls
    # one of the handle's own device, or an address that says nothing, is the caller's choice
    for call in calls:
        call(stream=Stream(1))
        call(stream=0x77)
    assert [a[-1] for _, a in seen.calls] == [0x7001, 0x77] * len(calls)
    current(monkeypatch, 1)
    for call in calls:
        call()
    assert [a[-1] for _, a in seen.calls[2 * len(calls):]] == [0x7001] * len(calls)
