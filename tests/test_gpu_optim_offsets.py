"""The norm and the step over a list whose tensors hold more than 2^31 values: fp32 and bf16 gradients, off alignment too.

Bounds as in tests/test_gpu_optim_lists.py: the norm and the coefficient are fp64 sums rounded to fp32 (2^-23), a step's
results go through at most 16 roundings of 2^-24 of their terms' magnitudes.  The norm's reference is a sum of fp64 sums; n
fp64 additions in any order are off by at most n 2^-53 of the sum, here 2^-21.9 for n = 2^31 in a row, far less in a tree, so
that both sums go over runs of at most 2^26: 2^-26 beside the rounding."""
import numpy as np
import pytest

import oracle
from gpu_support import say
from test_gpu_optim_lists import E, HYPER, _list, _norm

pytestmark = pytest.mark.gpu

RUN = 1 << 26


@pytest.mark.parametrize("bf16,shift", [(False, 0), (True, 3)])
def test_a_tensor_past_32_bits(bf16, shift):
    import paper_2609_33977_amd as gm
    import torch
    n = (1 << 31) + 8195
    say(f"a list of {n} and 77 values, {'bf16' if bf16 else 'fp32'} gradients {shift} off alignment (40 GB)")
    gen = torch.Generator(device="cuda").manual_seed(3)

    def values(scale, first, dtype=torch.float32):
        out = []
        for k in (n, 77):
            t = torch.empty(k + shift, dtype=dtype, device="cuda")[shift:]
            for i in range(0, k, RUN):
                part = t[i:i + RUN]
                part.copy_(first + scale * torch.rand(part.shape, generator=gen, device="cuda"))
            out.append(t)
        return out

    g = values(1e-3, 1e-3, torch.bfloat16 if bf16 else torch.float32)
    p, m, v = values(0.1, 1.0), values(0.0, 0.0), values(1e-6, 1e-6)
    p16 = values(0.0, 0.0, torch.bfloat16)
    total = sum(float(part.double().square().sum()) for t in g for part in t.split(RUN))
    want = total ** 0.5
    lst = _list(gm, g, p=p, m=m, v=v, p16=p16)
    norm, coef = _norm(gm, lst, 0.5 * want)
    k = 0.5
    assert abs(float(norm) - want) <= 2.0 ** -22.8 * want and abs(float(coef) - k) <= 2.0 ** -22.8 * k
    edges = (0, 8190, (1 << 31) - 100, n - 200)
    old = [[x[0][e:e + 200].double().cpu().numpy() for x in (p, g, m, v)] for e in edges]
    gm.gm_adamw_list(lst, coef=coef, **HYPER)
    torch.cuda.synchronize()
    c = float(coef)
    for e, (p0, g0, m0, v0) in zip(edges, old):
        P, M, V = oracle.adamw_step(p0, c * g0, m0, v0, **HYPER)
        root = np.sqrt(V / (1 - HYPER["beta2"] ** HYPER["step"])) + HYPER["eps"]
        magP = np.abs(p0) + HYPER["lr"] * np.abs(M) / (1 - HYPER["beta1"] ** HYPER["step"]) / root
        for what, got, ref, mag in (("m", m, M, np.abs(M)), ("v", v, V, V), ("p", p, P, magP)):
            off = np.abs(got[0][e:e + 200].double().cpu().numpy() - ref)
            assert np.all(off <= E * mag), (what, e, float(np.max(off - E * mag)))
    for i in range(2):                                     # every value was stepped, once: m = 0.1 c g with g in [1e-3, 2e-3]
        for at in range(0, g[i].numel(), RUN):
            got, grad = m[i][at:at + RUN], g[i][at:at + RUN].float()
            assert bool(((got / grad - 0.1 * c).abs() <= 2.0 ** -20 * 0.1 * c).all())
            assert torch.equal(p16[i][at:at + RUN], p[i][at:at + RUN].to(torch.bfloat16))
