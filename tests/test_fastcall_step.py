"""The extension module behind the calls over lists of tensors and rows of logits, on functions that record what they are called with: arguments arrive
in the header's structures, and what is not in a hot loop's form is left to ctypes (None, and no call)."""
import ctypes as C

import pytest
import torch

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S

vp, i32 = C.c_void_p, C.c_int32


class Tensor:
    """Stands for a device tensor."""
    def __init__(self, at, shape, dtype=torch.float32, strides=None, cuda=True):
        self.at, self.shape, self.dtype, self.is_cuda = at, tuple(shape), dtype, cuda
        self.strides = strides or tuple(torch.empty(shape, device="meta").stride())

    def stride(self):
        return self.strides

    def data_ptr(self):
        return self.at


def values(s):
    return {name: getattr(s, name) for name, _ in s._fields_}


@pytest.fixture
def calls():
    seen = []
    keep = [C.CFUNCTYPE(i32, vp, C.POINTER(S.McLogits), vp, vp)(lambda h, x, logp, st: seen.append((h, values(x[0]), logp, st)) or -7),
            C.CFUNCTYPE(i32, vp, C.POINTER(S.McLogits), C.POINTER(S.McPolicy), vp)(lambda h, x, p, st: seen.append((h, values(x[0]), values(p[0]), st)) or 3)]
    norm = C.CFUNCTYPE(i32, vp, C.c_float, C.c_float, vp, vp)
    keep += [norm(lambda *a: seen.append(("norm", *a)) or -1), norm(lambda *a: seen.append(("clip", *a)) or -2),
             C.CFUNCTYPE(i32, vp, C.POINTER(S.McAdamwConfig), vp, vp)(lambda h, c, coef, st: seen.append((h, values(c[0]), coef, st)) or 0)]
    fast = B._fastcall().StepCalls(torch.float32, torch.bfloat16, torch.float16, torch.int64, *[C.cast(k, vp).value for k in keep])
    return fast, seen, keep


def stream():
    return 0x7000


def good():
    rows, vocab = 5, 11
    return dict(logits=Tensor(2 ** 64 - 512, (rows, vocab), torch.bfloat16, (17, 1)), labels=Tensor(64, (rows,), torch.int64), old=Tensor(128, (rows,)),
                adv=Tensor(256, (rows,)), weights=Tensor(320, (rows,)), ref=Tensor(384, (rows,)), lo=0.25, hi=0.5, kl=0.125, temperature=0.75, scale=2.0,
                sums=Tensor(448, (8,)), logp=Tensor(512, (rows,)), dlogits=Tensor(1024, (rows, vocab), torch.bfloat16, (13, 1)))


def policy(fast, a, at=0xFFFF000000000010, stream=stream):
    return fast.policy_loss(at, a["logits"], a["labels"], a["old"], a["adv"], a["weights"], a["ref"], a["lo"], a["hi"], a["kl"], a["temperature"], a["scale"],
                            a["sums"], a["logp"], a["dlogits"], stream)


def test_arguments_arrive(calls):
    fast, seen, _ = calls
    a = good()
    x = dict(logits=2 ** 64 - 512, labels=64, rows=5, vocab=11, stride=17, dtype=1, temperature=0.75)
    assert policy(fast, a) == 3
    assert seen[-1] == (0xFFFF000000000010, x, dict(old_logp=128, advantages=256, weights=320, ref_logp=384, clip_low=0.25, clip_high=0.5, kl_coef=0.125,
                                                    grad_scale=2.0, sums=448, logp=512, dlogits=1024, dlogits_stride=13), 0x7000)
    a.update(weights=None, ref=None, logp=None, dlogits=None)
    assert policy(fast, a) == 3
    assert seen[-1][2] == dict(old_logp=128, advantages=256, weights=None, ref_logp=None, clip_low=0.25, clip_high=0.5, kl_coef=0.125, grad_scale=2.0,
                               sums=448, logp=None, dlogits=None, dlogits_stride=0)
    for number, kind in enumerate((torch.float32, torch.bfloat16, torch.float16)):
        raw = B._fastcall().RawStream(lambda d: 0x100 + d, lambda: 3)
        assert fast.token_logp(8, Tensor(16, (3, 9), kind), Tensor(32, (3,), torch.int64), Tensor(48, (3,)), 1.0, raw) == -7
        assert seen[-1] == (8, dict(logits=16, labels=32, rows=3, vocab=9, stride=9, dtype=number, temperature=1.0), 48, 0x103)
    # one row: how far the next would be does not matter, but never less than a row
    assert fast.token_logp(8, Tensor(16, (1, 9), strides=(1, 1)), Tensor(32, (1,), torch.int64), Tensor(48, (1,)), 1.0, stream) == -7
    assert seen[-1][1]["stride"] == 9


def test_same_layout_as_ctypes(calls):
    """What _rows says of a tensor's layout is what arrives."""
    fast, seen, _ = calls
    for x in (torch.empty(4, 6), torch.empty(4, 9)[:, 2:8], torch.empty(1, 6), torch.empty(1, 6).expand(1, 6), torch.empty(6, 1).t(), torch.empty(3, 1), torch.empty(0, 6)):
        t = Tensor(16, x.shape, x.dtype, x.stride())
        assert S._rows(t, "x") == (x.shape[0], x.shape[1], fast.token_logp(8, t, Tensor(32, (x.shape[0],), torch.int64), Tensor(48, (x.shape[0],)), 1.0, stream) and
                                   seen[-1][1]["stride"])


def test_other_forms_are_left_to_ctypes(calls):
    fast, seen, _ = calls
    wrong = dict(logits=[Tensor(16, (5, 11), torch.float64), Tensor(16, (5, 11), strides=(1, 5)), Tensor(16, (5, 11), cuda=False), Tensor(16, (55,)), None, 3],
                 labels=[Tensor(16, (5,), torch.int32), Tensor(16, (4,), torch.int64), Tensor(16, (5,), torch.int64, (2,)), None],
                 old=[None, Tensor(16, (6,)), Tensor(16, (5, 1)), Tensor(16, (5,), torch.float16), Tensor(16, (5,), cuda=False)],
                 adv=[None, Tensor(16, (5,), torch.int64)], weights=[Tensor(16, (1,)), Tensor(16, (5,), torch.bool), 1.0], ref=[Tensor(16, (5,), strides=(0,))],
                 lo=[1, None], hi=[torch.tensor(0.2)], kl=[0], temperature=[1], scale=["2"], sums=[None, Tensor(16, (7,)), Tensor(16, (8,), torch.int32)],
                 logp=[Tensor(16, (4,))], dlogits=[Tensor(16, (5, 11)), Tensor(16, (5, 10), torch.bfloat16), Tensor(16, (5, 11), torch.bfloat16, (1, 5))])
    for name, bad in wrong.items():
        for value in bad:
            assert policy(fast, {**good(), name: value}) is None, (name, value)
    assert policy(fast, good(), at="8") is None and policy(fast, good(), stream=None) is None and policy(fast, good(), stream=lambda: None) is None
    assert fast.policy_loss(8) is None and fast.token_logp() is None
    assert not seen


def test_lists(calls):
    fast, seen, _ = calls
    out, one = Tensor(64, (2,)), Tensor(80, (1,))
    assert fast.grad_norm(8, 0.5, 2.0, out, stream) == -1 and seen[-1] == ("norm", 8, 0.5, 2.0, 64, 0x7000)
    assert fast.grad_clip(8, 0.5, float("inf"), out, stream) == -2 and seen[-1] == ("clip", 8, 0.5, float("inf"), 64, 0x7000)
    cfg = dict(lr=0.1, beta1=0.2, beta2=0.3, eps=0.4, weight_decay=0.5, step=2 ** 40)
    assert fast.adamw(8, 2 ** 40, 0.1, 0.2, 0.3, 0.4, 0.5, one, stream) == 0 and seen[-1] == (8, cfg, 80, 0x7000)
    assert fast.adamw(8, 2 ** 40, 0.1, 0.2, 0.3, 0.4, 0.5, None, stream) == 0 and seen[-1] == (8, cfg, None, 0x7000)
    before = len(seen)
    for bad in ((8, 1, 2.0, out, stream), (8, 0.5, None, out, stream), (8, 0.5, 2.0, one, stream), (8, 0.5, 2.0, None, stream), (8, 0.5, 2.0, out, None),
                (8, 0.5, 2.0, Tensor(64, (2,), torch.float64), stream), (None, 0.5, 2.0, out, stream), (8, 0.5)):
        assert fast.grad_norm(*bad) is None and fast.grad_clip(*bad) is None, bad
    for bad in ((8, 1.0, 0.1, 0.2, 0.3, 0.4, 0.5, one, stream), (8, 2 ** 70, 0.1, 0.2, 0.3, 0.4, 0.5, one, stream), (8, 1, 0.1, 0.2, 0.3, 0.4, 0, one, stream),
                (8, 1, 0.1, 0.2, 0.3, 0.4, 0.5, out, stream), (8, 1, 0.1, 0.2, 0.3, 0.4, 0.5, one, None), (8, 1)):
        assert fast.adamw(*bad) is None, bad
    assert len(seen) == before
