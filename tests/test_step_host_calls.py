"""The host code of the operators in mergecomp_step.h without a device: step_api.hip linked with tests/host/no_device.hip, whose allocator counts
(and refuses beyond a limit), and launchers that note their calls.  No kernel runs here."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import build as hip_build
from paper_2103_15195_amd import step as S

HERE = os.path.dirname(os.path.abspath(__file__))
NO_LIMIT = 2 ** 64 - 1
vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("step"))
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    objects, jobs = [], []
    for src in (os.path.join(hip_build.CSRC, "step_api.hip"), os.path.join(HERE, "host", "no_device.hip"), os.path.join(HERE, "host", "no_device_step.hip")):
        objects.append(os.path.join(out, os.path.basename(src) + ".o"))
        jobs.append(subprocess.Popen([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "-c", *flags, "-o", objects[-1], src],
                                     stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for job in jobs:
        text, _ = job.communicate()
        assert job.returncode == 0, text
    path = os.path.join(out, "libstep.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,defs", "-o", path, *objects], check=True)
    L = C.CDLL(path)
    L.nd_reset.argtypes = [C.c_size_t]
    L.nd_held.restype = C.c_size_t
    L.nd_denied.restype = L.nd_bad_free.restype = C.c_long
    L.nds_log.restype = C.c_char_p
    L.mc_step_create.argtypes = [C.POINTER(vp), vp, i32, i32, i32, vp]
    L.mc_step_destroy.argtypes = L.mc_loss_destroy.argtypes = [vp]
    L.mc_step_bind.argtypes = [vp, i32, vp, vp]
    L.mc_grad_norm.argtypes = L.mc_grad_clip.argtypes = [vp, f32, f32, vp, vp]
    L.mc_adamw.argtypes = [vp, C.POINTER(S.McAdamwConfig), vp, vp]
    L.mc_loss_create.argtypes = [C.POINTER(vp)]
    L.mc_token_logp.argtypes = [vp, C.POINTER(S.McLogits), vp, vp]
    L.mc_policy_loss.argtypes = [vp, C.POINTER(S.McLogits), C.POINTER(S.McPolicy), vp]
    return L


@pytest.fixture
def host(lib):
    lib.nd_reset(NO_LIMIT)
    lib.nds_forget()
    held = lib.nd_held()
    yield lib
    assert lib.nd_held() == held and lib.nd_bad_free() == 0


def log(L):
    text = L.nds_log().decode().split()
    L.nds_forget()
    return text


def step_of(L, sizes, grad=0, model=-1):
    h = vp()
    return L.mc_step_create(C.byref(h), (C.c_int64 * len(sizes))(*sizes), len(sizes), grad, model, None), h


def addresses(*at):
    return (vp * len(at))(*at)


def test_nothing_is_left_behind_when_memory_runs_out(host):
    """Refused at every allocation in turn: the status says so, no handle, and all that was there is given back."""
    sizes = [100000, 0, 7]
    before = host.nd_held()
    for make, destroy in ((lambda h: host.mc_step_create(C.byref(h), (C.c_int64 * 3)(*sizes), 3, 0, -1, None), host.mc_step_destroy),
                          (lambda h: host.mc_loss_create(C.byref(h)), host.mc_loss_destroy)):
        h = vp()
        assert make(h) == B.MC_OK
        need = host.nd_held() - before
        assert destroy(h) == B.MC_OK and host.nd_held() == before
        denied = 0
        for limit in range(0, need, max(1, need // 50)):
            host.nd_reset(before + limit)
            h = vp()
            assert make(h) == B.MC_ERR_ALLOC and not h.value
            assert host.nd_held() == before
            denied += host.nd_denied()
        assert denied
        host.nd_reset(NO_LIMIT)


def test_pieces_cover_a_tensor_wherever_it_begins(host):
    """Elements and 63 more (of 16 bits, in a line of 128 bytes) in pieces of 4096."""
    for n in (0, 1, 4033, 4034, 4096, 4097, 8129, 8130, 100000):
        rc, h = step_of(host, [n])
        assert rc == B.MC_OK
        assert host.mc_step_bind(h, 0, addresses(64 if n else None), None) == B.MC_OK
        assert host.mc_grad_norm(h, 1.0, 1.0, 64, None) == B.MC_OK
        assert log(host) == [f"norm:{(n + 63 + 4095) // 4096 if n else 0}"]
        assert host.mc_step_destroy(h) == B.MC_OK


def test_lists(host):
    """What has to be bound, in what alignment, and what a call consists of."""
    rc, h = step_of(host, [10, 0, 5], grad=1, model=2)
    assert rc == B.MC_OK
    cfg = S.McAdamwConfig(1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    assert host.mc_grad_norm(h, 1.0, 1.0, 64, None) == B.MC_ERR_INVALID_ARG
    assert host.mc_step_bind(h, 0, addresses(2, None, 6), None) == B.MC_OK                  # 16 bits: even addresses
    assert host.mc_step_bind(h, 0, addresses(3, None, 6), None) == B.MC_ERR_INVALID_ARG
    assert host.mc_step_bind(h, 0, addresses(2, 2, None), None) == B.MC_ERR_INVALID_ARG
    assert host.mc_step_bind(h, 0, None, None) == B.MC_ERR_INVALID_ARG
    for out in (0, 2, 65):
        assert host.mc_grad_norm(h, 1.0, 1.0, out or None, None) == B.MC_ERR_INVALID_ARG
    assert host.mc_grad_clip(h, 1.0, 1.0, 64, None) == B.MC_OK and log(host) == ["norm:2", "clip:0"]
    assert host.mc_step_bind(h, 1, addresses(2, None, 6), None) == B.MC_OK
    assert host.mc_grad_clip(h, 1.0, 1.0, 64, None) == B.MC_OK and log(host) == ["norm:2", "clip:1"]
    for which in (2, 3, 4):
        assert host.mc_adamw(h, C.byref(cfg), None, None) == B.MC_ERR_INVALID_ARG
        assert host.mc_step_bind(h, which, addresses(2, None, 4), None) == B.MC_ERR_INVALID_ARG      # 32 bits
        assert host.mc_step_bind(h, which, addresses(8, None, 4), None) == B.MC_OK
    assert host.mc_adamw(h, C.byref(cfg), None, None) == B.MC_ERR_INVALID_ARG
    assert host.mc_step_bind(h, 5, addresses(2, None, 4), None) == B.MC_OK
    assert host.mc_adamw(h, C.byref(cfg), 2, None) == B.MC_ERR_INVALID_ARG
    assert log(host) == []
    assert host.mc_adamw(h, C.byref(cfg), 4, None) == B.MC_OK and log(host) == ["adamw+copy:2"]
    assert host.mc_adamw(h, None, None, None) == B.MC_ERR_INVALID_ARG
    for at in (-1, 6):
        assert host.mc_step_bind(h, at, addresses(8, None, 4), None) == B.MC_ERR_INVALID_ARG
    assert host.mc_step_destroy(h) == B.MC_OK
    rc, h = step_of(host, [10])
    assert host.mc_step_bind(h, 5, addresses(8), None) == B.MC_ERR_INVALID_ARG               # made without a copy
    assert host.mc_step_destroy(h) == B.MC_OK


def test_a_list_without_elements(host):
    rc, h = step_of(host, [0, 0])
    cfg = S.McAdamwConfig(1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    assert rc == B.MC_OK and host.mc_grad_clip(h, 1.0, 1.0, 64, None) == host.mc_adamw(h, C.byref(cfg), None, None) == B.MC_OK
    assert host.mc_step_bind(h, 0, addresses(None, None), None) == B.MC_OK
    assert host.mc_step_destroy(h) == B.MC_OK


def test_rows(host):
    h = vp()
    assert host.mc_loss_create(C.byref(h)) == B.MC_OK
    x = dict(logits=256, labels=512, rows=4, vocab=10, stride=12, dtype=1, temperature=1.0)
    p = dict(old_logp=64, advantages=64, weights=None, ref_logp=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, grad_scale=1.0, sums=64, logp=None,
             dlogits=1024, dlogits_stride=10)

    def policy(**k):
        return host.mc_policy_loss(h, C.byref(S.McLogits(**{**x, **{a: v for a, v in k.items() if a in x}})),
                                   C.byref(S.McPolicy(**{**p, **{a: v for a, v in k.items() if a in p}})), None)

    def logp(at=64, **k):
        return host.mc_token_logp(h, C.byref(S.McLogits(**{**x, **k})), at, None)
    assert policy() == logp() == B.MC_OK and log(host) == ["policy:4", "logp:4"]
    inf, nan = float("inf"), float("nan")
    both = [dict(rows=-1), dict(vocab=0), dict(stride=9), dict(dtype=3), dict(dtype=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=inf),
            dict(temperature=nan), dict(temperature=1e-40), dict(logits=None), dict(labels=None), dict(logits=257), dict(labels=516)]
    for k in both:
        assert policy(**k) == logp(**k) == B.MC_ERR_INVALID_ARG, k
    for k in (dict(rows=2 ** 31), dict(vocab=2 ** 31 - 2 ** 16, stride=2 ** 31)):
        assert policy(**k, dlogits_stride=2 ** 31) == logp(**k) == B.MC_ERR_RANGE, k
    for k in (dict(old_logp=None), dict(advantages=None), dict(sums=None), dict(old_logp=66), dict(weights=65), dict(ref_logp=66), dict(logp=3), dict(sums=66),
              dict(dlogits=1025), dict(dlogits_stride=9), dict(dlogits=256), dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_high=-0.1), dict(clip_high=inf),
              dict(clip_low=nan), dict(kl_coef=-1.0), dict(kl_coef=inf), dict(grad_scale=nan), dict(grad_scale=3e38, temperature=1e-3)):
        assert policy(**k) == B.MC_ERR_INVALID_ARG, k
    assert logp(at=None) == logp(at=66) == B.MC_ERR_INVALID_ARG
    assert log(host) == []
    assert policy(dlogits=256, dlogits_stride=12) == policy(dlogits=None, dlogits_stride=0) == policy(rows=0, logits=None, labels=None, old_logp=None,
                                                                                                     advantages=None, dlogits=None) == B.MC_OK
    assert logp(at=None, rows=0, logits=None, labels=None) == B.MC_OK
    assert host.mc_loss_destroy(h) == B.MC_OK
