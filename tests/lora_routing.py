"""Routings with a stated number of tokens per adapter, and bounds by adapter, for the adapters' tests."""
from __future__ import annotations

import numpy as np

from lora_support import make, references


def routed(counts, n, d_in, widths, r, none=0, seed=1):
    """A case whose adapter k has counts[k] tokens (the rest of the n none), `none` tokens without one, in any order."""
    T = sum(counts) + none
    c = make(T, n, d_in, widths, r, "none", seed)
    ids = np.concatenate([np.repeat(np.arange(len(counts)), counts), np.full(none, -1)])
    c.ids[:] = np.random.default_rng(seed).permutation(ids)
    return c


def references_by_adapter(oracle, c, P=None):
    """lora_support's references, with dB's bound by the adapter's own tokens: its sums go over t of them, so
    (3 t + 16) u sum |products|, as dA's do."""
    ref = references(oracle, c, P)
    value, bound = ref["dB"]
    t = np.bincount(c.ids[(c.ids >= 0) & (c.ids < c.n)], minlength=c.n)
    ref["dB"] = (value, bound * ((3 * t + 16) / (3 * c.T + 16))[:, None, None])
    return ref
