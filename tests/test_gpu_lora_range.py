"""Adapters whose finite P and Q lie past the largest bf16 value, 255 2^120: their first bf16 term may not round to
infinity.  Bounds: those of tests/lora_support.py, which are relative, and for products below the normal numbers of fp32
(2^-126), which these inputs have, the absolute ones beside them:
  an fp32 operation is off by at most one step there, D = 2^-149, so a sum of K products by K D;
  a bf16 term's step is 2^-133 there, so what a value's terms leave of it is at most half of that, S = 2^-134, whatever
  their number.  Both reach Y, dX and dA through the products that follow, by the weights' (rows') magnitudes."""
import numpy as np
import pytest

import oracle
from gpu_support import say
from lora_support import backward, check, f64, forward, make, references

pytestmark = pytest.mark.gpu

MOST = 255 * 2.0 ** 120
PAST = MOST + 1.5 * 2.0 ** 119   # rounds to 2^128 in bf16, finite in fp32


def _case(T, few, r, sign):
    """Adapter 1 has the tokens of `few`, of which the first has P[3] = sign PAST and Q[5] = PAST (c = 1)."""
    import torch
    c = make(T, 2, 64, (72,), r, "all")
    tiny = 2.0 ** -100
    c.ids[few] = 1
    c.scale[1] = 1.0
    for t in (c.A, c.B):
        t[1] *= tiny
    c.A[1, 3, 0], c.A[1, 3, 1] = sign * MOST, sign * 1.5 * 2.0 ** 119
    c.B[1, 0, 5], c.B[1, 1, 5] = MOST, 1.5 * 2.0 ** 119
    c.X[few] *= 2.0 ** -30            # the sums over tokens stay within fp32
    c.dY[few] *= 2.0 ** -30
    c.X[few[0], :2] = 1.0
    c.dY[few[0], :2] = 1.0
    assert all(torch.isfinite(t.float()).all() for t in (c.A, c.B, c.X, c.dY))
    return c


D, S = 2.0 ** -149, 2.0 ** -134


def _below_normal(c):
    """{name: bound} of what operations below the normal numbers add."""
    X, A, B, scale = (np.abs(f64(t)) for t in (c.X, c.A, c.B, c.scale))
    a = np.maximum(c.ids, 0)                               # every token has an adapter here
    low, high = c.d_in * D, c.d_out * D                    # P, and dY B
    q = scale[a] * high + D                                # Q, per token
    Y = B.sum(2)[a] * (scale[a] * low + D + S)[:, None] + (2 * c.r + 4) * D
    dX = A.sum(1)[a] * (q + S)[:, None] + (2 * c.R + 4) * D
    dA = np.stack([((q + S)[c.ids == k, None] * X[c.ids == k]).sum(0) for k in range(c.n)])[:, None] + (3 * c.T + 16) * D
    dY = np.abs(f64(c.dY))
    dB = np.stack([(S * scale[k] * dY[c.ids == k]).sum(0) for k in range(c.n)])[:, :, None] + (3 * c.T + 16) * D
    return {"P": low, "Y": Y, "dX": dX, "dA": dA, "dB": dB}


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T,count,r", [(3, 1, 16), (60, 20, 16), (60, 50, 64), (60, 40, 24), (30, 9, 72)])
def test_values_past_the_largest_bf16(T, count, r, sign):
    import paper_2609_33977_amd as gm
    say(f"adapters: P = {sign * PAST:g}, Q = {PAST:g}; {count} of {T} tokens in its adapter, r={r}")
    c = _case(T, np.arange(T - count, T), r, sign)
    Y, P = forward(gm, c)
    assert f64(P)[T - count, 3] == sign * PAST          # two products, their sum exact in fp32
    ref = references(oracle, c, P)
    dX, dA, dB = backward(gm, c, P)
    more = _below_normal(c)
    for name, got in (("Y", Y), ("P", P), ("dX", dX), ("dA", dA), ("dB", dB)):
        check(name, got, (ref[name][0], ref[name][1] + more[name]))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_infinities_and_nan_still_reach_their_rows(bad):
    import paper_2609_33977_amd as gm
    import torch
    say(f"adapters: a token's X and dY hold {bad}")
    c = make(60, 2, 64, (72,), 16, "all")
    c.ids[40:] = 1
    c.X[45, 7] = c.dY[45, 9] = bad
    Y, P = forward(gm, c)
    dX, dA, dB = backward(gm, c, P)
    sick = torch.zeros(60, dtype=torch.bool)
    sick[45] = True
    for t in (Y, P, dX):
        t = t.cpu().float()
        assert not torch.isfinite(t[sick]).any() and torch.isfinite(t[~sick]).all()
    for t in (dA, dB):
        t = t.cpu()
        assert not torch.isfinite(t[1]).all() and torch.isfinite(t[0]).all()
