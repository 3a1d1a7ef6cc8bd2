"""mc_adamw's hyperparameters are given in 64 bits and used in 32: what is no use there is refused.  The host code without a device, as in
test_step_host_calls.py; no kernel runs here."""
import ctypes as C

import pytest

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S
from test_step_host_calls import addresses, host, lib, log, step_of  # noqa: F401  (fixtures)

GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=3)


@pytest.fixture
def update(host):
    rc, h = step_of(host, [10])
    assert rc == B.MC_OK
    for which in (0, 2, 3, 4):
        assert host.mc_step_bind(h, which, addresses(64), None) == B.MC_OK
    yield lambda **k: host.mc_adamw(h, C.byref(S.McAdamwConfig(**{**GOOD, **k})), None, None)
    assert host.mc_step_destroy(h) == B.MC_OK


def test_what_is_no_number_in_32_bits_is_refused(update, host):
    for k in (dict(eps=1e-46), dict(eps=5e-324), dict(eps=1e39), dict(eps=1e300), dict(lr=1e39), dict(lr=1e300, weight_decay=0.0),
              dict(lr=1e38, beta1=0.99, step=1), dict(lr=1.0, weight_decay=1e39), dict(lr=1e30, weight_decay=1e30), dict(lr=1e300, weight_decay=1e300)):
        assert update(**k) == B.MC_ERR_INVALID_ARG, k
    assert log(host) == []


def test_what_is_one_is_taken(update, host):
    """Also where it is of little use: below binary32's normal numbers, next to 1, or far on."""
    taken = [{}, dict(eps=1e-44), dict(eps=1e38), dict(lr=0.0), dict(lr=1e-300), dict(lr=1e37, weight_decay=0.0), dict(weight_decay=0.0), dict(beta1=0.0, beta2=0.0),
             dict(beta1=1.0 - 2.0 ** -53, beta2=1.0 - 2.0 ** -53, step=1), dict(step=2 ** 62)]
    for k in taken:
        assert update(**k) == B.MC_OK, k
    assert log(host) == ["adamw:1"] * len(taken)
