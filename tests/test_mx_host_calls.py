"""The host code of the operators in mergecomp_mx.h without a device: mx_api.hip linked with tests/host/no_device.hip, whose allocator counts
(and refuses beyond a limit), and launchers that note their calls.  No kernel runs here."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import build as hip_build
from paper_2103_15195_amd import mx as X
from paper_2103_15195_amd import step as S

HERE = os.path.dirname(os.path.abspath(__file__))
NO_LIMIT = 2 ** 64 - 1
BAD, RANGE = B.MC_ERR_INVALID_ARG, B.MC_ERR_RANGE
vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("mx"))
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    objects, jobs = [], []
    for src in (os.path.join(hip_build.CSRC, "mx_api.hip"), os.path.join(HERE, "host", "no_device.hip"), os.path.join(HERE, "host", "no_device_mx.hip")):
        objects.append(os.path.join(out, os.path.basename(src) + ".o"))
        jobs.append(subprocess.Popen([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "-c", *flags, "-o", objects[-1], src],
                                     stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for job in jobs:
        text, _ = job.communicate()
        assert job.returncode == 0, text
    path = os.path.join(out, "libmx.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,defs", "-o", path, *objects], check=True)
    L = C.CDLL(path)
    L.nd_reset.argtypes = [C.c_size_t]
    L.nd_held.restype = C.c_size_t
    L.nd_denied.restype = L.nd_bad_free.restype = C.c_long
    L.ndm_log.restype = C.c_char_p
    L.mc_step8_create.argtypes = [C.POINTER(vp), vp, i32, i32, i32, vp]
    L.mc_step8_destroy.argtypes = L.mc_mx_destroy.argtypes = [vp]
    L.mc_step8_bind.argtypes = [vp, i32, vp, vp]
    L.mc_adamw8.argtypes = [vp, C.POINTER(S.McAdamwConfig), vp, vp]
    for f in (L.mc_mx_code_bytes, L.mc_mx_scale_bytes):
        f.argtypes, f.restype = [i64, i64], C.c_size_t
    L.mc_mx_create.argtypes = [C.POINTER(vp)]
    L.mc_mx_quantize.argtypes = [vp, C.POINTER(X.McMxSource), C.POINTER(X.McMxMatrix), C.POINTER(X.McMxMatrix), vp, i64, vp]
    L.mc_mx_matmul.argtypes = [vp, C.POINTER(X.McMxMatrix), C.POINTER(X.McMxMatrix), C.POINTER(X.McMxResult), vp]
    return L


@pytest.fixture
def host(lib):
    lib.nd_reset(NO_LIMIT)
    lib.ndm_forget()
    held = lib.nd_held()
    yield lib
    assert lib.nd_held() == held and lib.nd_bad_free() == 0


@pytest.fixture
def mx(host):
    h = vp()
    assert host.mc_mx_create(C.byref(h)) == B.MC_OK
    yield h
    assert host.mc_mx_destroy(h) == B.MC_OK


def log(L):
    text = L.ndm_log().decode().split()
    L.ndm_forget()
    return text


def addresses(*at):
    return (vp * len(at))(*at)


def test_nothing_is_left_behind_when_memory_runs_out(host):
    sizes = [100000, 0, 7]
    before = host.nd_held()
    for make, destroy in ((lambda h: host.mc_step8_create(C.byref(h), (i64 * 3)(*sizes), 3, 0, -1, None), host.mc_step8_destroy),
                          (lambda h: host.mc_mx_create(C.byref(h)), host.mc_mx_destroy)):
        h = vp()
        assert make(h) == B.MC_OK
        need = host.nd_held() - before
        assert destroy(h) == B.MC_OK and host.nd_held() == before
        denied = 0
        for limit in range(0, need, max(1, need // 50)):
            host.nd_reset(before + limit)
            h = vp()
            assert make(h) == B.MC_ERR_ALLOC and not h.value and host.nd_held() == before
            denied += host.nd_denied()
        assert denied
        host.nd_reset(NO_LIMIT)


def test_lists(host):
    """What has to be bound, in what alignment, and what a call consists of."""
    h = vp()
    cfg = S.McAdamwConfig(1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    for wrong in ((0, 3, 0, -1), (0, 1, 3, -1), (0, 1, 0, 0), (-1, 1, 0, -1)):
        assert host.mc_step8_create(C.byref(h), (i64 * 1)(wrong[0]), 0 if wrong[1] == 3 else 1, wrong[2], wrong[3], None) == BAD
    assert host.mc_step8_create(C.byref(h), (i64 * 1)(2 ** 39), 1, 0, -1, None) == RANGE
    assert host.mc_step8_create(None, (i64 * 1)(1), 1, 0, -1, None) == host.mc_step8_create(C.byref(h), None, 1, 0, -1, None) == BAD
    assert host.mc_step8_create(C.byref(h), (i64 * 3)(2049, 0, 5), 3, 1, 2, None) == B.MC_OK
    align = {0: 2, 1: 4, 2: 2, 3: 1, 4: 1, 5: 4, 6: 4}
    for which, a in align.items():
        assert host.mc_adamw8(h, C.byref(cfg), None, None) == BAD
        if a > 1:
            assert host.mc_step8_bind(h, which, addresses(8 * a + a // 2, None, 8), None) == BAD
        assert host.mc_step8_bind(h, which, addresses(8, None, None), None) == BAD
        assert host.mc_step8_bind(h, which, addresses(8 + a, None, 8), None) == B.MC_OK
    assert host.mc_adamw8(h, C.byref(cfg), 2, None) == host.mc_adamw8(h, None, None, None) == host.mc_adamw8(None, C.byref(cfg), None, None) == BAD
    assert log(host) == []
    assert host.mc_adamw8(h, C.byref(cfg), 4, None) == B.MC_OK and log(host) == ["adamw8+copy:3"]
    for at in (-1, 7):
        assert host.mc_step8_bind(h, at, addresses(8, None, 4), None) == BAD
    assert host.mc_step8_destroy(h) == B.MC_OK
    assert host.mc_step8_create(C.byref(h), (i64 * 2)(0, 0), 2, 0, -1, None) == B.MC_OK
    assert host.mc_step8_bind(h, 2, addresses(8, 8), None) == BAD                               # made without a copy
    assert host.mc_adamw8(h, C.byref(cfg), None, None) == B.MC_OK and log(host) == ["adamw8:0"]
    assert host.mc_step8_destroy(h) == B.MC_OK


def test_sizes(host):
    for rows, cols in ((0, 1), (1, 1), (16, 128), (17, 129), (64, 256), (65, 300), (2 ** 31 - 2 ** 16 - 1, 5)):
        steps = -(-cols // 128)
        assert host.mc_mx_code_bytes(rows, cols) == -(-rows // 16) * steps * 1024
        assert host.mc_mx_scale_bytes(rows, cols) == -(-rows // 64) * steps * 256
    for rows, cols in ((-1, 5), (5, 0), (5, -1), (2 ** 31, 5), (5, 2 ** 31 - 2 ** 16)):
        assert host.mc_mx_code_bytes(rows, cols) == host.mc_mx_scale_bytes(rows, cols) == 0


M = 1 << 20                                  # places that lie far from each other


def matrix(at, rows, cols, **k):
    return X.McMxMatrix(**{**dict(codes=at, scales=at + M // 2, rows=rows, cols=cols), **k})


def test_quantize(host, mx):
    def call(src=None, r="r", c="c", v=None, vs=0, **k):
        x = X.McMxSource(**{**dict(data=64 * M, rows=20, cols=50, stride=60, dtype=1), **k}) if src is None else src
        rows, cols = (matrix(80 * M, 20, 50) if r == "r" else r), (matrix(90 * M, 50, 20) if c == "c" else c)
        return host.mc_mx_quantize(mx, C.byref(x), None if rows is None else C.byref(rows), None if cols is None else C.byref(cols), v, vs, None)
    assert call() == call(c=None) == call(r=None) == call(v=70 * M, vs=50) == call(r=None, c=None, v=70 * M, vs=51) == B.MC_OK
    assert log(host) == ["quantize:20x50r1c1", "quantize:20x50r1", "quantize:20x50c1", "quantize:20x50r1c1v", "quantize:20x50v"]
    assert call(v=64 * M, vs=60) == B.MC_OK and log(host) == ["quantize:20x50r1c1v"]           # in place
    for k in (dict(rows=-1), dict(cols=0), dict(stride=49), dict(dtype=3), dict(dtype=-1), dict(data=None), dict(data=64 * M + 1), dict(r=None, c=None),
              dict(v=70 * M, vs=49), dict(v=70 * M + 1, vs=50), dict(v=64 * M, vs=61), dict(v=64 * M + 2, vs=60),
              dict(r=matrix(80 * M, 50, 20)), dict(c=matrix(90 * M, 20, 50)), dict(r=matrix(80 * M, 20, 51)), dict(r=matrix(80 * M + 8, 20, 50)),
              dict(r=matrix(80 * M, 20, 50, scales=81 * M + 2)), dict(r=matrix(80 * M, 20, 50, codes=None)), dict(r=matrix(64 * M + 96, 20, 50)),
              dict(c=matrix(80 * M, 50, 20)), dict(c=matrix(80 * M + M // 2, 50, 20)), dict(v=80 * M, vs=50), dict(r=matrix(80 * M, 20, 50, scales=80 * M + 1024))):
        assert call(**k) == BAD, k
    assert call(rows=2 ** 31) == call(cols=2 ** 31, stride=2 ** 31) == RANGE
    assert host.mc_mx_quantize(None, None, None, None, None, 0, None) == host.mc_mx_quantize(mx, None, None, None, None, 0, None) == BAD
    assert log(host) == []
    assert call(rows=0, data=None, r=matrix(0, 0, 50, codes=None, scales=None), c=None) == B.MC_OK and log(host) == []


def test_matmul(host, mx):
    def call(a=None, b=None, **k):
        y = X.McMxResult(**{**dict(out=64 * M, stride=30, dtype=1, accumulate=0, bias=None), **k})
        return host.mc_mx_matmul(mx, C.byref(a or matrix(80 * M, 20, 300)), C.byref(b or matrix(90 * M, 30, 300)), C.byref(y), None)
    assert call() == call(bias=70 * M, accumulate=1) == B.MC_OK
    assert log(host) == ["matmul:20x30x3", "matmul:20x30x3b+"]
    for k in (dict(out=None), dict(out=64 * M + 1), dict(stride=29), dict(dtype=3), dict(dtype=-1), dict(bias=70 * M + 2), dict(a=matrix(80 * M, 20, 301)),
              dict(a=matrix(80 * M, -1, 300)), dict(a=matrix(80 * M, 20, 0)), dict(a=matrix(80 * M + 8, 20, 300)), dict(b=matrix(90 * M, 30, 300, scales=None)),
              dict(out=80 * M), dict(out=80 * M + M // 2), dict(out=90 * M + 1022), dict(bias=64 * M), dict(out=70 * M, bias=70 * M + 20 * 60 - 4)):
        assert call(**k) == BAD, k
    assert call(a=matrix(80 * M, 2 ** 31, 300)) == call(b=matrix(80 * M, 2 ** 31, 300)) == call(a=matrix(80 * M, 20, 2 ** 31), b=matrix(90 * M, 30, 2 ** 31)) == RANGE
    assert host.mc_mx_matmul(mx, None, None, None, None) == BAD and log(host) == []
    nothing = X.McMxMatrix(None, None, 0, 300)
    assert call(a=nothing, out=None) == call(b=nothing, out=None) == B.MC_OK and log(host) == []
