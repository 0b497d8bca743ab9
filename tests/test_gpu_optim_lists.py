"""The gradient norm, the clipping coefficient and AdamW over lists of tensors against the fp64 oracle.

Bounds: squares and sums are fp64, so the norm and the coefficient carry their one rounding to fp32 (2^-24; 2^-23 with
the fp64 sum's order).  A step's fp32 result goes through at most 16 roundings of 2^-24: the moments are sums of two
products (their terms' magnitudes times 2^-21), and the parameter moves by lr |m^| / (sqrt(v^) + eps), whose terms'
magnitudes count once more."""
import numpy as np
import pytest

import oracle
from gpu_support import say

pytestmark = pytest.mark.gpu

E = 2.0 ** -20  # 16 roundings
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=3)


def _make(sizes, seed=1, bf16=(), shift=0):
    """Tensors of the given sizes in one buffer per role, `shift` values off alignment."""
    import torch
    g = torch.Generator().manual_seed(seed)

    def role(std, dtype=torch.float32, positive=False):
        out = []
        for k in sizes:
            t = torch.randn(k + shift, generator=g) * std
            out.append((t.abs() + 1e-6 if positive else t).to(dtype).cuda()[shift:])
        return out

    grads = [t.to(torch.bfloat16) if i in bf16 else t for i, t in enumerate(role(0.1))]
    if shift:
        grads = [torch.cat([t.new_zeros(shift), t])[shift:] for t in grads]
    return grads, role(1.0), role(0.1), role(0.01, positive=True), [t[shift:] for t in
                                                                    (torch.zeros(k + shift, dtype=torch.bfloat16, device="cuda") for k in sizes)]


def _list(gm, grads, **rest):
    import torch
    lst = torch.empty(gm.gm_tensor_list_size([t.numel() for t in grads]), dtype=torch.uint8, device="cuda")
    gm.gm_tensor_list(grads, lst, **rest)
    return lst


def _norm(gm, lst, max_norm):
    import torch
    norm, coef = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    ws = torch.empty(gm.GM_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    gm.gm_grad_norm(lst, max_norm, norm, coef, ws)
    torch.cuda.synchronize()
    return norm, coef


def _h(ts):
    return [t.double().cpu().numpy() for t in ts]


LISTS = [([1], (), 0), ([0, 5, 0], (), 0), ([8191, 8192, 8193], (), 0), ([3, 100000, 7, 16385], (1, 2), 0),
         ([40, 8200], (), 1), ([40, 8200, 9001], (0, 2), 3), ([17] * 200, tuple(range(0, 200, 3)), 0),
         ([5_000_001], (), 0), ([30_000_000, 11], (1,), 0)]


@pytest.mark.parametrize("sizes,bf16,shift", LISTS)
def test_norm_and_step(sizes, bf16, shift):
    import paper_2609_33977_amd as gm
    import torch
    say(f"list of {len(sizes)} tensors, first {sizes[:4]}, {len(bf16)} bf16 gradients, {shift} off alignment")
    g, p, m, v, p16 = _make(sizes, bf16=bf16, shift=shift)
    want, _ = oracle.grad_norm(_h(g), 1.0)
    lst = _list(gm, g, p=p, m=m, v=v, p16=p16)
    for max_norm in (0.5 * want, 2 * want, float("inf")):
        norm, coef = _norm(gm, lst, max_norm)
        k = oracle.grad_norm(_h(g), max_norm)[1]
        assert abs(float(norm) - want) <= 2.0 ** -23 * want and abs(float(coef) - k) <= 2.0 ** -23 * k
    old, kept = [_h(x) for x in (p, m, v)], [t.clone() for t in g]
    norm, coef = _norm(gm, lst, 0.5 * want)
    gm.gm_adamw_list(lst, coef=coef, **HYPER)
    torch.cuda.synchronize()
    c = float(coef)
    for i in range(len(sizes)):
        gi = _h([kept[i]])[0]
        assert torch.equal(g[i], kept[i])
        P, M, V = oracle.adamw_step(old[0][i], c * gi, old[1][i], old[2][i], **HYPER)
        magM = 0.9 * np.abs(old[1][i]) + 0.1 * np.abs(c * gi)
        root = np.sqrt(V / (1 - 0.99 ** 3)) + 1e-8
        magP = np.abs(old[0][i]) + 1e-2 * magM / (1 - 0.9 ** 3) / root
        for what, got, ref, mag in (("m", m, M, magM), ("v", v, V, V), ("p", p, P, magP)):
            off = np.abs(_h([got[i]])[0] - ref)
            assert np.all(off <= E * mag + 1e-44), (what, i, float(np.max(off - E * mag)))
        assert torch.equal(p16[i], p[i].to(torch.bfloat16))


def test_step_without_coefficient_is_the_flat_step():
    import paper_2609_33977_amd as gm
    import torch
    g, p, m, v, _ = _make([10007])
    q = [t[0].clone() for t in (p, m, v)]
    gm.gm_adamw_list(_list(gm, g, p=p, m=m, v=v), **HYPER)
    gm.gm_adamw(q[0], g[0], q[1], q[2], HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["weight_decay"],
                HYPER["step"])
    torch.cuda.synchronize()
    for a, b in zip((p[0], m[0], v[0]), q):
        assert float((a - b).abs().max()) <= E * float(b.abs().max())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_gradients_that_are_not_finite_change_nothing(value):
    import paper_2609_33977_amd as gm
    import torch
    g, p, m, v, p16 = _make([9000, 20])
    g[1][3] = value
    lst = _list(gm, g, p=p, m=m, v=v, p16=p16)
    old = [t.clone() for x in (p, m, v, p16) for t in x]
    norm, coef = _norm(gm, lst, 1.0)
    assert float(coef) == 0.0 and not np.isfinite(float(norm))
    gm.gm_adamw_list(lst, coef=coef, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(old, [t for x in (p, m, v, p16) for t in x]))


def test_squares_past_the_range_of_fp32():
    import paper_2609_33977_amd as gm
    import torch
    for value, count in ((1e30, 1000), (1e-30, 1000), (3e38, 1)):
        g = [torch.full((count,), value, device="cuda")]
        norm, coef = _norm(gm, _list(gm, g), 1.0)
        want = float(np.float32(value)) * count ** 0.5
        k = min(1.0, 1.0 / want)
        assert abs(float(norm) - want) <= 2.0 ** -22 * want
        assert abs(float(coef) - k) <= 2.0 ** -22 * k + 1e-45
    g = [torch.full((16,), 3e38, device="cuda")]      # finite gradients whose norm is past fp32
    norm, coef = _norm(gm, _list(gm, g), 1.0)
    assert float(norm) == float("inf") and 0.0 <= float(coef) < 1e-38
    zero = [torch.zeros(100, device="cuda")]
    norm, coef = _norm(gm, _list(gm, zero), 1.0)
    assert float(norm) == 0.0 and float(coef) == 1.0


def test_only_gradients_and_repeats():
    import paper_2609_33977_amd as gm
    import torch
    g, *_ = _make([100003, 77, 5000], bf16=(2,))
    lst = _list(gm, g)
    a, b = _norm(gm, lst, 1.0), _norm(gm, lst, 1.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    gm.gm_adamw_list(lst, coef=a[1], **HYPER)          # nothing to step
    torch.cuda.synchronize()


def test_a_gradient_twice_counts_twice():
    import paper_2609_33977_amd as gm
    g, *_ = _make([9001])
    norm, _ = _norm(gm, _list(gm, [g[0], g[0], g[0][1:]]), 1.0)
    h = _h([g[0], g[0], g[0][1:]])
    want = oracle.grad_norm(h, 1.0)[0]
    assert abs(float(norm) - want) <= 2.0 ** -23 * want


def test_something_that_is_no_list_is_not_followed():
    import paper_2609_33977_amd as gm
    import torch
    junk = torch.full((4096,), 7, dtype=torch.uint8, device="cuda")
    norm, coef = _norm(gm, junk, 1.0)
    assert float(norm) == 0.0 and float(coef) == 1.0
    gm.gm_adamw_list(junk, **HYPER)
    torch.cuda.synchronize()


def test_captured_step_follows_its_buffers():
    import paper_2609_33977_amd as gm
    import torch
    g, p, m, v, p16 = _make([9000, 333])
    lst = _list(gm, g, p=p, m=m, v=v, p16=p16)
    norm, coef = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(gm.GM_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def step():
        gm.gm_grad_norm(lst, 1.0, norm, coef, ws)
        gm.gm_adamw_list(lst, coef=coef, **HYPER)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state = [t for x in (p, m, v, p16) for t in x]
    for i in range(3):
        for t in g:
            t.copy_(torch.randn(t.numel(), generator=torch.Generator().manual_seed(i)).to(t.dtype))
        before = [t.clone() for t in state]
        graph.replay()
        torch.cuda.synchronize()
        after = [t.clone() for t in state]
        for t, o in zip(state, before):
            t.copy_(o)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(after, state)) and not torch.equal(before[0], after[0])
