"""Inputs of the low-rank adapters' tests, the library's calls on them, and error bounds derived from the number formats.

Bounds (all against the fp64 oracle on the same bf16 inputs).  u = 2^-23 covers one fp32 operation of a sum whatever
its rounding (to nearest or towards zero), so a sum of K products of values is off by at most K u sum |products|.
  P, Q      K u sum |x||a| with K = the contracted length
  terms     c P and Q enter a bf16 result with two bf16 terms: 2^-8 2^-8 = 2^-16 of the value, and one rounding of c P
  Y, dX     the error of P or Q times |weights|, 2^-16 and 2 r + 2 fp32 operations of the product, then one rounding
            to bf16, half a step of which is 2^-8 of the value
  dA, dB    the error of Q (given P) times |rows|, then T + 8 fp32 operations of the sum over tokens in three terms, and
            the scale: (3 T + 16) u sum |products|
"""
from __future__ import annotations

import dataclasses

import numpy as np

U, HALF16, TERMS = 2.0 ** -23, 2.0 ** -8, 2.0 ** -16


@dataclasses.dataclass
class Case:
    T: int
    n: int
    d_in: int
    widths: tuple
    r: int
    ids: np.ndarray
    X: object
    A: object
    B: object
    scale: object
    base: object
    dY: object
    dXb: object

    @property
    def d_out(self):
        return sum(self.widths)

    @property
    def R(self):
        return self.r * len(self.widths)


def f64(t):
    return t.detach().cpu().double().numpy()


def ids_of(kind, T, n, seed):
    """Adapters of T tokens: 'mixed' draws with some -1, 'runs' of one adapter, 'none', 'all' (adapter 0), 'bad' with
    values far outside the pool among them."""
    rng = np.random.default_rng((seed, T, n))
    if kind == "none":
        ids = np.full(T, -1)
    elif kind == "all":
        ids = np.zeros(T)
    elif kind == "runs":
        ids = np.sort(rng.integers(0, n, T))[np.argsort(rng.integers(0, 2, T), kind="stable")]
    else:
        ids = rng.integers(0, n, T)
        ids[rng.random(T) < 0.2] = -1
        if kind == "bad":
            odd = rng.random(T) < 0.3
            ids[odd] = rng.choice(np.array([n, n + 1, -5, 2 ** 31 - 1, -2 ** 31]), int(odd.sum()))
    return ids.astype(np.int32)


def make(T, n, d_in, widths, r, kind="mixed", seed=1):
    import torch
    g = torch.Generator().manual_seed(7919 * seed + 31 * T + d_in)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16)

    d_out, R = sum(widths), r * len(widths)
    return Case(T, n, d_in, tuple(widths), r, ids_of(kind, T, n, seed), normal(T, d_in),
                normal(n, R, d_in, std=d_in ** -0.5), normal(n, d_out, r, std=0.5 * r ** -0.5),
                0.5 + torch.rand(n, generator=g), normal(T, d_out), normal(T, d_out, std=0.1), normal(T, d_in, std=0.1))


def plan_of(gm, ids, n):
    import torch
    t = ids if isinstance(ids, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(ids)).cuda()
    plan = torch.empty(gm.gm_lora_plan_size(t.numel(), n), dtype=torch.uint8, device="cuda")
    gm.gm_lora_plan(t, n, plan)
    return plan


def space(gm, op, c):
    import torch
    return torch.empty(max(16, gm.gm_lora_workspace_size(op, c.T, c.n, c.d_in, c.widths, c.r)), dtype=torch.uint8,
                       device="cuda")


def forward(gm, c, plan=None, keep=True):
    import torch
    plan = plan_of(gm, c.ids, c.n) if plan is None else plan
    Y = torch.full((c.T, c.d_out), 3.0, dtype=torch.bfloat16, device="cuda")
    P = torch.full((c.T, c.R), 3.0, device="cuda") if keep else None
    gm.gm_lora_fwd(c.X.cuda(), c.A.cuda(), c.B.cuda(), c.scale.cuda(), plan, c.base.cuda(), Y, P, space(gm, gm.GM_OP_FWD, c),
                   widths=c.widths)
    torch.cuda.synchronize()
    return Y, P


def backward(gm, c, P, plan=None):
    import torch
    plan = plan_of(gm, c.ids, c.n) if plan is None else plan
    dX = torch.full((c.T, c.d_in), 3.0, dtype=torch.bfloat16, device="cuda")
    dA, dB = torch.full(c.A.shape, 3.0, device="cuda"), torch.full(c.B.shape, 3.0, device="cuda")
    gm.gm_lora_bwd(c.dY.cuda(), c.X.cuda(), c.A.cuda(), c.B.cuda(), c.scale.cuda(), plan, P.cuda(), c.dXb.cuda(), dX, dA, dB,
                   space(gm, gm.GM_OP_BWD, c), widths=c.widths)
    torch.cuda.synchronize()
    return dX, dA, dB


def references(oracle, c, P=None):
    """The oracle's results and the bounds of each: {name: (value, bound)}."""
    X, A, B, scale, base, dY, dXb = (f64(t) for t in (c.X, c.A, c.B, c.scale, c.base, c.dY, c.dXb))
    Y, P64 = oracle.lora_fwd(X, A, B, scale, c.ids, base, c.widths)
    kept = P64 if P is None else f64(P)
    dX, dA, dB, Q = oracle.lora_bwd(dY, X, A, B, scale, c.ids, dXb, kept, c.widths)
    one = np.ones_like(scale)
    absX, absA, absB, absdY = (np.abs(v) for v in (X, A, B, dY))

    def fwd(low, factor):  # sum over a part's ranks of |low| |B|, by the oracle's own indexing
        out = np.zeros((c.T, c.d_out))
        edges = np.concatenate([[0], np.cumsum(c.widths)])
        for a in range(c.n):
            t = np.flatnonzero(c.ids == a)
            for k in range(len(c.widths)):
                o = slice(int(edges[k]), int(edges[k + 1]))
                out[t, o] = factor[a] * (low[t][:, k * c.r:(k + 1) * c.r] @ absB[a, o].T)
        return out

    _, Pabs = oracle.lora_fwd(absX, absA, absB, one, c.ids, np.zeros_like(base), c.widths)
    eP = c.d_in * U * Pabs
    mag = fwd(np.abs(P64), scale)
    eY = fwd(eP, scale) + (TERMS + (2 * c.r + 4) * U) * mag + 2 * U * np.abs(base)
    zeros = np.zeros_like(dXb)
    magX, _, _, Qabs = oracle.lora_bwd(absdY, absX, absA, absB, scale, c.ids, zeros, np.abs(kept), c.widths)
    eQ = (max(c.widths) + 2) * U * Qabs
    exX, exA, exB = zeros.copy(), np.zeros_like(dA), np.zeros_like(dB)
    for a in range(c.n):
        t = np.flatnonzero(c.ids == a)
        exX[t] = eQ[t] @ absA[a] + (TERMS + (2 * c.R + 4) * U) * (np.abs(Q[t]) @ absA[a]) + 2 * U * np.abs(dXb[t])
        exA[a] = eQ[t].T @ absX[t] + (3 * t.size + 16) * U * (np.abs(Q[t]).T @ absX[t])
    _, _, magB, _ = oracle.lora_bwd(absdY, absX, absA, absB, scale, c.ids, zeros, np.abs(kept), c.widths)
    exB = (3 * c.T + 16) * U * magB
    rounded = lambda v, e: e + HALF16 * (np.abs(v) + e)  # noqa: E731
    return {"Y": (Y, rounded(Y, eY)), "P": (P64, eP), "dX": (dX, rounded(dX, exX)), "dA": (dA, exA), "dB": (dB, exB)}


def check(what, got, ref):
    value, bound = ref
    off = np.abs(f64(got) - value)
    worst = float(np.max(off - bound))
    assert np.all(np.isfinite(f64(got))) and worst <= 0.0, \
        f"{what}: off by {worst:.3e} beyond its bound at {np.unravel_index(np.argmax(off - bound), off.shape)}"
