"""Host side of the operators in mergecomp_step.h: what the library exports, what it refuses before it touches a device, and
what the binding refuses.  No kernel is launched here."""
import ctypes as C
import os
import re

import pytest
import torch

import step_reference as R
from paper_2103_15195_amd import binding as B
from paper_2103_15195_amd import step as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mergecomp_step.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(mc_[a-z_0-9]+)\s*\(", text)))
    assert declared == sorted(S.EXPORTS)
    assert all(hasattr(S.lib(), name) for name in declared)


def test_create_refuses_before_it_touches_a_device():
    L, h = S.lib(), C.c_void_p()

    def create(sizes, grad=0, model=-1, count=None):
        n = (C.c_int64 * len(sizes))(*sizes)
        return L.mc_step_create(C.byref(h), n, len(sizes) if count is None else count, grad, model, None)
    assert L.mc_step_create(None, (C.c_int64 * 1)(1), 1, 0, -1, None) == B.MC_ERR_INVALID_ARG
    assert L.mc_step_create(C.byref(h), None, 1, 0, -1, None) == B.MC_ERR_INVALID_ARG
    assert create([4], count=0) == B.MC_ERR_INVALID_ARG and create([4, -1]) == B.MC_ERR_INVALID_ARG
    for grad in (-1, 3):
        assert create([4], grad=grad) == B.MC_ERR_INVALID_ARG
    for model in (0, 3, -2):
        assert create([4], model=model) == B.MC_ERR_INVALID_ARG
    assert create([2 ** 43]) == B.MC_ERR_RANGE and create([2 ** 42, 2 ** 42]) == B.MC_ERR_RANGE
    assert h.value is None
    assert L.mc_loss_create(None) == B.MC_ERR_INVALID_ARG


def test_no_handle_is_refused():
    L = S.lib()
    x, p, c = S.McLogits(), S.McPolicy(), S.McAdamwConfig()
    assert L.mc_step_destroy(None) == L.mc_loss_destroy(None) == B.MC_ERR_INVALID_ARG
    assert L.mc_step_bind(None, 0, (C.c_void_p * 1)(16), None) == B.MC_ERR_INVALID_ARG
    assert L.mc_grad_norm(None, 1.0, 1.0, 16, None) == L.mc_grad_clip(None, 1.0, 1.0, 16, None) == B.MC_ERR_INVALID_ARG
    assert L.mc_adamw(None, C.byref(c), None, None) == B.MC_ERR_INVALID_ARG
    assert L.mc_token_logp(None, C.byref(x), 16, None) == L.mc_policy_loss(None, C.byref(x), C.byref(p), None) == B.MC_ERR_INVALID_ARG


def test_structures_have_the_header_s_layout():
    assert C.sizeof(S.McAdamwConfig) == 48 and C.sizeof(S.McLogits) == 48 and C.sizeof(S.McPolicy) == 80
    assert S.McPolicy.sums.offset == 48 and S.McLogits.dtype.offset == 40 and S.McAdamwConfig.step.offset == 40


def test_binding_refuses_what_is_no_list_of_the_model():
    for wrong in (dict(grad_dtype=torch.float64), dict(grad_dtype=torch.int8), dict(model_dtype=torch.float32), dict(no_decay=[True])):
        with pytest.raises(ValueError):
            S.Step([3, 4], **wrong)
    assert S.dtype_id(torch.bfloat16) == S.dtype_id("bfloat16") == S.MC_DTYPE_BF16 and S.dtype_id(None) == S.MC_DTYPE_NONE


@pytest.mark.parametrize("kl", [0.0, 0.2])
def test_reference_gradient_against_differences(kl):
    """The definition's gradient, as the tests on the GPU use it, by central differences in 64 bits: of every logit."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(5, 7, generator=gen, dtype=torch.float64)
    labels = torch.tensor([0, 6, 3, -100, 2])
    adv, w = torch.randn(5, generator=gen), torch.tensor([0.5, 1.0, 0.25, 1.0, 0.0])
    base = torch.log_softmax(x / 0.7, 1)[torch.arange(5), labels.clamp(min=0)]
    old = base - torch.tensor([0.4, -0.1, -0.4, 0.0, 0.0])
    ref = base + 0.5 if kl else None
    kw = dict(clip=(0.2, 0.3), kl_coef=kl, temperature=0.7)
    got = R.Policy(x, labels, old, adv, w, ref, grad_scale=3.0, **kw).dlogits
    h = 2.0 ** -12
    for i in range(5):
        for j in range(7):
            e = torch.zeros_like(x)
            e[i, j] = h
            d = (R.Policy(x + e, labels, old, adv, w, ref, **kw).sums[0] - R.Policy(x - e, labels, old, adv, w, ref, **kw).sums[0]) / (2 * h)
            assert abs(3.0 * d - float(got[i, j])) <= 100 * h * h


def test_reference_adamw_against_torch():
    """The definition, as the tests on the GPU use it, against torch.optim.AdamW in 64 bits over several steps."""
    gen = torch.Generator().manual_seed(4)
    p = torch.randn(50, generator=gen, dtype=torch.float64)
    q = torch.nn.Parameter(p.clone())
    opt = torch.optim.AdamW([q], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    for t in range(1, 6):
        g = torch.randn(50, generator=gen, dtype=torch.float64)
        q.grad = 0.5 * g
        opt.step()
        (p, m, v), _ = R.adamw(p, m, v, g, 0.5, t, 1e-2, (0.9, 0.95), 1e-8, 0.1)
        assert bool(((p - q.detach()).abs() <= 1e-12).all())
