"""What the calls over rows of logits write may not lie over what they read: a row's blocks and wavefronts read and write it in no order.  The host code
without a device, as in test_step_host_calls.py; no kernel runs here."""
import ctypes as C

import pytest

from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S
from test_step_host_calls import host, lib, log, vp  # noqa: F401  (fixtures)

ROWS, VOCAB, STRIDE = 5, 10, 16
# bytes: each of them far from the others
AT = dict(logits=0x1000, labels=0x2000, old_logp=0x3000, advantages=0x4000, weights=0x5000, ref_logp=0x6000, sums=0x7000, logp=0x8000, dlogits=0x9000)
BYTES = dict(labels=8 * ROWS, old_logp=4 * ROWS, advantages=4 * ROWS, weights=4 * ROWS, ref_logp=4 * ROWS, sums=32, logp=4 * ROWS)


class Loss:
    def __init__(self, lib):
        self.lib, self.h = lib, vp()
        assert lib.mc_loss_create(C.byref(self.h)) == B.MC_OK

    def _rows(self, k, dtype):
        return S.McLogits(k["logits"], k["labels"], k.get("rows", ROWS), k.get("vocab", VOCAB), k.get("stride", STRIDE), dtype, 1.0)

    def policy(self, dtype=0, **k):
        k = {**AT, **k}
        p = S.McPolicy(k["old_logp"], k["advantages"], k["weights"], k["ref_logp"], 0.2, 0.2, 0.1, 1.0, k["sums"], k["logp"], k["dlogits"], k.get("dstride", STRIDE))
        return self.lib.mc_policy_loss(self.h, C.byref(self._rows(k, dtype)), C.byref(p), None)

    def token(self, dtype=0, **k):
        k = {**AT, **k}
        return self.lib.mc_token_logp(self.h, C.byref(self._rows(k, dtype)), k["logp"], None)


@pytest.fixture
def loss(host):
    it = Loss(host)
    yield it
    assert host.mc_loss_destroy(it.h) == B.MC_OK


READ = ["labels", "old_logp", "advantages", "weights", "ref_logp"]


@pytest.mark.parametrize("name", READ)
def test_log_probabilities_over_what_is_read(loss, host, name):
    at, n = AT[name], BYTES[name]
    for where in (at, at + 4, at + n - 4, at - BYTES["logp"] + 4):
        assert loss.policy(logp=where) == B.MC_ERR_INVALID_ARG, hex(where)
        if name == "labels":
            assert loss.token(logp=where) == B.MC_ERR_INVALID_ARG
    assert log(host) == []
    for where in (at + n, at - BYTES["logp"]):
        assert loss.policy(logp=where) == B.MC_OK
    assert loss.policy(logp=None) == B.MC_OK
    # two that are read may be the same
    assert loss.policy(old_logp=AT["ref_logp"]) == loss.policy(advantages=AT["weights"]) == B.MC_OK


def test_vectors_over_rows(loss, host):
    """A vector may lie in what is between two rows, and nowhere on one."""
    first, step, row = AT["logits"], 4 * STRIDE, 4 * VOCAB
    for where in (first, first + row - 4, first - 4, first + step - 4, first + (ROWS - 1) * step + row - 4, first + 2 * step):
        assert loss.policy(logp=where) == loss.token(logp=where) == B.MC_ERR_INVALID_ARG, hex(where)
        shifted = where - first + AT["dlogits"]
        assert loss.policy(logp=shifted) == loss.policy(sums=shifted) == B.MC_ERR_INVALID_ARG
        for name in READ:
            if shifted % 8 == 0 or name != "labels":
                assert loss.policy(**{name: shifted}) == B.MC_ERR_INVALID_ARG, name
    assert log(host) == []
    assert step - row >= BYTES["logp"]
    for where in (first + row, first + step + row, first + (ROWS - 1) * step + row, first - BYTES["logp"]):
        assert loss.policy(logp=where) == loss.token(logp=where) == B.MC_OK
    assert loss.policy(logp=AT["dlogits"] + row) == B.MC_OK


def test_sums(loss):
    for where in (AT["logp"], AT["logp"] - 28, AT["logp"] + 4 * ROWS - 4):
        assert loss.policy(sums=where) == B.MC_ERR_INVALID_ARG
    assert loss.policy(sums=AT["logp"] + 4 * ROWS) == loss.policy(sums=AT["logp"] - 32) == B.MC_OK
    # with more rows than are taken at a time, sums are written before the last rows are read
    many = 2 ** 17 + 1
    far = {name: at << 20 for name, at in AT.items()}
    assert loss.policy(**far, rows=many) == B.MC_OK
    for name in READ + ["logits"]:
        assert loss.policy(**{**far, "sums": far[name]}, rows=many) == B.MC_ERR_INVALID_ARG, name


def test_gradient_over_logits(loss, host):
    x, step, row = AT["logits"], 4 * STRIDE, 4 * VOCAB
    for where in (x + 4, x + row - 4, x + step, x + step - row + 4, x - row + 4, x + (ROWS - 1) * step, x - (ROWS - 1) * step):
        assert loss.policy(dlogits=where) == B.MC_ERR_INVALID_ARG, hex(where)
    for where, dstride in ((x + 8, 12), (x, 12), (x - 4, 40), (x + 2 * step, 32)):
        assert loss.policy(dlogits=where, dstride=dstride) == B.MC_ERR_INVALID_ARG
    assert loss.policy(dlogits=x + 4, rows=1) == loss.policy(dlogits=x + 4, rows=1, dstride=10) == B.MC_ERR_INVALID_ARG
    assert log(host) == []
    assert loss.policy(dlogits=x) == B.MC_OK                                            # the logits themselves
    assert loss.policy(dlogits=x + ROWS * step) == loss.policy(dlogits=x - ROWS * step) == loss.policy(dlogits=x + (ROWS - 1) * step + row) == B.MC_OK
    # columns of one buffer, rows of one buffer
    assert loss.policy(dlogits=x + row, stride=2 * VOCAB, dstride=2 * VOCAB) == loss.policy(dlogits=x + step, stride=2 * STRIDE, dstride=2 * STRIDE) == B.MC_OK
    assert loss.policy(dlogits=x + row, stride=4 * VOCAB, dstride=8 * VOCAB) == B.MC_OK
    assert loss.policy(dlogits=x + step, rows=1) == B.MC_OK
    assert loss.policy(dtype=1, dlogits=x + 2 * VOCAB, stride=2 * VOCAB, dstride=2 * VOCAB) == B.MC_OK
    assert loss.policy(dtype=1, dlogits=x + 2 * VOCAB - 2, stride=2 * VOCAB, dstride=2 * VOCAB) == B.MC_ERR_INVALID_ARG


def test_no_rows_and_far_apart(loss):
    assert loss.policy(rows=0, logp=AT["old_logp"], dlogits=AT["logits"] + 4) == loss.token(rows=0, logp=AT["labels"]) == B.MC_OK
    # strides whose products pass 64 bits
    for stride in (2 ** 61, 2 ** 62, 2 ** 63 - 1):
        assert loss.policy(stride=stride, dstride=stride, rows=1) == B.MC_OK
        assert loss.policy(stride=stride, rows=1, logp=AT["logits"] + 8) == B.MC_ERR_INVALID_ARG
