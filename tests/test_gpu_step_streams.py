"""The operators in mergecomp_step.h with a stream handed over, which goes through ctypes, against the same calls on torch's current stream."""
import pytest
import torch

from paper_2103_15195_amd import step as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("form", ["stream", "handle"])
def test_same_results_on_a_stream_of_ones_own(form):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    numel = [70001, 3, 4096]

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)
    x, labels = normal(50, 3001), torch.randint(0, 3001, (50,), device=DEV, generator=gen)
    adv, weights, first = normal(50), torch.rand(50, device=DEV, generator=gen), [[normal(n) for n in numel] for _ in range(3)]
    first[2] = [v.square() for v in first[2]]
    g = [normal(n) for n in numel]
    torch.cuda.synchronize()
    results = []
    for stream in (None, torch.cuda.Stream()):
        p, m, v = ([t.clone() for t in l] for l in first)
        norm, logp, ref, sums, slopes, clipped = (torch.zeros(2, device=DEV), torch.zeros(50, device=DEV), torch.zeros(50, device=DEV), torch.zeros(8, device=DEV),
                                                  torch.zeros_like(x), [torch.zeros_like(t) for t in g])
        torch.cuda.synchronize()                 # all of it is there for the other stream
        on = stream if form == "stream" or stream is None else stream.cuda_stream
        h, loss = S.Step(numel), S.PolicyLoss()
        h.bind(stream=on, grads=g, clipped=clipped, params=p, exp_avg=m, exp_avg_sq=v)
        h.mc_grad_norm(1.0, norm, stream=on)
        h.mc_grad_clip(0.5, norm, stream=on)
        h.mc_adamw(3, 1e-2, (0.9, 0.95), 1e-8, 0.1, coef=norm[1:], stream=on)
        loss.mc_token_logp(x, labels, ref, 0.8, stream=on)
        loss.mc_policy_loss(x, labels, ref, adv, weights=weights, ref_logp=ref, kl_coef=0.1, temperature=0.9, sums=sums, logp=logp, dlogits=slopes, stream=on)
        torch.cuda.synchronize()
        results.append([norm, ref, logp, sums, slopes, *clipped, *p, *m, *v])
        h.close()
        loss.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert float(results[0][0][0]) > 1 and bool(results[0][4].any())
