"""Handing over lists of tensors, with a recorder in the library's place: what arrives there, and what is kept, whatever kind of iterable
a list comes in.  Needs no device."""
import ctypes as C

import pytest
import torch

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S


class Recorder:
    """Stands for the loaded library; notes the addresses that arrive, as many as the array holds."""

    def __init__(self, status=B.MC_OK):
        self.seen, self.status = [], status

    def mc_step_bind(self, handle, which, ptrs, stream):
        self.seen.append((which, [p for p in ptrs], stream))
        return self.status

    def mc_strerror(self, status):
        return b"refused"


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(S, "lib", lambda: r)
    monkeypatch.setattr(B, "lib", lambda: r)
    return r


def step_of(numel):
    """A handle's Python side alone, for tensors in host memory."""
    h = S.Step.__new__(S.Step)
    h.numel = list(numel)
    h.dtypes = {"grads": S.MC_DTYPE_BF16, "clipped": S.MC_DTYPE_BF16, "model": S.MC_DTYPE_F16, "params": S.MC_DTYPE_F32, "exp_avg": S.MC_DTYPE_F32,
                "exp_avg_sq": S.MC_DTYPE_F32}
    h._kept, h._h, h._at, h._fast, h._device = {}, None, 0, None, torch.device("cpu")
    return h


KINDS = {"list": list, "tuple": tuple, "generator": lambda l: (t for t in l), "iterator": iter, "parameters": lambda l: torch.nn.ParameterList(l).parameters(),
         "map": lambda l: map(lambda t: t, l)}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("numel", [[5, 3, 7], [0, 3, 7], [4]])
def test_every_kind_of_iterable_arrives_whole(recorder, numel, kind):
    h = step_of(numel)
    tensors = [torch.nn.Parameter(torch.zeros(n)) for n in numel]
    h.bind(stream=0x70, params=KINDS[kind](tensors))
    assert recorder.seen == [(S.LISTS["params"], [t.data_ptr() or None for t in tensors], 0x70)]
    assert [id(t) for t in h._kept["params"]] == [id(t) for t in tensors]


def test_several_generators_in_one_call(recorder):
    numel = [0, 4, 9]
    h = step_of(numel)
    lists = {name: [torch.zeros(n, dtype=kind) for n in numel] for name, kind in (("grads", torch.bfloat16), ("params", torch.float32), ("model", torch.float16))}
    h.bind(stream=0, **{name: (t for t in l) for name, l in lists.items()})
    assert recorder.seen == [(S.LISTS[name], [t.data_ptr() or None for t in l], 0) for name, l in lists.items()]
    assert {name: [id(t) for t in l] for name, l in h._kept.items()} == {name: [id(t) for t in l] for name, l in lists.items()}


def test_one_wrong_list_leaves_all_as_they_were(recorder):
    h = step_of([4, 9])
    good = [torch.zeros(4), torch.zeros(9)]
    h.bind(stream=0, params=good)
    for bad in ([torch.zeros(4)], [torch.zeros(4), torch.zeros(8)], [torch.zeros(4), torch.zeros(9).double()], [torch.zeros(8)[::2], torch.zeros(9)]):
        with pytest.raises(ValueError):
            h.bind(stream=0, exp_avg=iter(good), params=iter(bad))
    with pytest.raises(ValueError):
        h.bind(stream=0, exp_avg=iter(good), weights=iter(good))
    assert len(recorder.seen) == 1 and h._kept == {"params": good}
    recorder.status = B.MC_ERR_DEVICE
    with pytest.raises(B.McError):
        h.bind(stream=0, exp_avg=iter(good))
    assert h._kept == {"params": good}
