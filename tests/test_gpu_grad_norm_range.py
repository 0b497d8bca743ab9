"""The clipping coefficient at the ends of fp32's range: it is 0 where the norm that is returned is not finite, and only
there, so that a step is skipped for such a norm and for no other.

Bounds: the squares' sum, its root and the quotient are fp64; the norm and the coefficient are then rounded to fp32 (2^-24
each, and the least positive value, 2^-149, in the place of a smaller coefficient)."""
import numpy as np
import pytest

from gpu_support import say
from test_gpu_optim_lists import HYPER, _list, _norm

pytestmark = pytest.mark.gpu

LEAST, MOST = 2.0 ** -149, float(np.finfo(np.float32).max)


def _state(gm, g):
    import torch
    p, m, v = ([torch.full_like(t, x, dtype=torch.float32) for t in g] for x in (1.0, 0.5, 0.25))
    p16 = [torch.zeros_like(t, dtype=torch.bfloat16) for t in g]
    return _list(gm, g, p=p, m=m, v=v, p16=p16), [p, m, v, p16]


@pytest.mark.parametrize("max_norm", [1e-10, 1.0, 1e30, float("inf")])
@pytest.mark.parametrize("value,count", [(3e38, 16), (3e38, 9000), (MOST, 2)])
def test_a_norm_past_fp32_steps_nothing(value, count, max_norm):
    import paper_2609_33977_amd as gm
    import torch
    say(f"{count} gradients of {value:g}, clipped to {max_norm:g}")
    g = [torch.full((count,), value, device="cuda")]
    lst, state = _state(gm, g)
    old = [t.clone() for ts in state for t in ts]
    norm, coef = _norm(gm, lst, max_norm)
    assert float(norm) == float("inf") and float(coef) == 0.0
    gm.gm_adamw_list(lst, coef=coef, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(old, [t for ts in state for t in ts]))


@pytest.mark.parametrize("value,count,max_norm", [(1e38, 1, 1e-10), (MOST, 1, 1e-10), (1e38, 9, 1e-30), (MOST, 1, 1.0),
                                                  (1e30, 4, 1e-12), (1e-40, 4, 1.0), (2.0, 4, 1e-38)])
def test_a_finite_norm_always_steps(value, count, max_norm):
    import paper_2609_33977_amd as gm
    import torch
    say(f"{count} gradients of {value:g}, clipped to {max_norm:g}")
    g = [torch.full((count,), value, device="cuda")]
    lst, state = _state(gm, g)
    norm, coef = _norm(gm, lst, max_norm)
    exact = float(np.float32(value)) * count ** 0.5
    assert abs(float(norm) - exact) <= 2.0 ** -23 * exact + LEAST / 2
    want = max(min(1.0, float(np.float32(max_norm)) / exact), LEAST)
    # half a step of fp32 (2^-24 of the value, 2^-150 below the normal numbers), and the fp64 operations before it
    assert 0.0 < float(coef) and abs(float(coef) - want) <= 2.0 ** -23.9 * want + 2.0 ** -149.9
    gm.gm_adamw_list(lst, coef=coef, **HYPER)
    torch.cuda.synchronize()
    m, clipped = state[1][0].double().cpu().numpy(), float(coef) * float(np.float32(value))
    exact_m = HYPER["beta1"] * 0.5 + (1 - HYPER["beta1"]) * clipped
    assert np.all(np.abs(m - exact_m) <= 2.0 ** -21 * (0.5 + abs(clipped)))     # the moment decayed: a step was made
