"""fp64 oracle of the low-rank adapters and of the clipped optimiser step (NumPy only, token by token's adapter).

Shapes as in the library's header: A [n, parts r, d_in], B [n, d_out, r], widths of the stacked parts."""
from __future__ import annotations

import numpy as np


def _parts(widths, r):
    """(rank slice, output slice) of every part."""
    edges = np.concatenate([[0], np.cumsum(widths)])
    return [(slice(k * r, (k + 1) * r), slice(int(edges[k]), int(edges[k + 1]))) for k in range(len(widths))]


def lora_fwd(X, A, B, scale, adapter, base, widths):
    """(Y, P)."""
    n, R, _ = A.shape
    P = np.zeros((X.shape[0], R))
    Y = np.array(base, dtype=np.float64)
    for a in range(n):
        t = np.flatnonzero(adapter == a)
        if t.size == 0:
            continue
        P[t] = X[t] @ A[a].T
        for ranks, outs in _parts(widths, B.shape[2]):
            Y[t, outs] += scale[a] * (P[t, ranks] @ B[a, outs].T)
    return Y, P


def lora_bwd(dY, X, A, B, scale, adapter, base, P, widths):
    """(dX, dA, dB, Q)."""
    n, R, _ = A.shape
    Q = np.zeros((X.shape[0], R))
    dX, dA, dB = np.array(base, dtype=np.float64), np.zeros(A.shape), np.zeros(B.shape)
    for a in range(n):
        t = np.flatnonzero(adapter == a)
        if t.size == 0:
            continue
        for ranks, outs in _parts(widths, B.shape[2]):
            Q[t, ranks] = scale[a] * (dY[t, outs] @ B[a, outs])
            dB[a, outs] = scale[a] * (dY[t, outs].T @ P[t, ranks])
        dX[t] += Q[t] @ A[a]
        dA[a] = Q[t].T @ X[t]
    return dX, dA, dB, Q


def grad_norm(grads, max_norm: float):
    """(norm, clipping coefficient) of a sequence of arrays; the coefficient is 0 where the norm is not finite."""
    norm = float(np.sqrt(sum(float(np.sum(np.square(np.asarray(g, dtype=np.float64)))) for g in grads)))
    if not np.isfinite(norm):
        return norm, 0.0
    return norm, (max_norm / norm if norm > max_norm else 1.0)
