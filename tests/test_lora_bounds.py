"""The bounds of the adapters' gradients tell a token that is missing or counted twice, at the largest batch too."""
import numpy as np
import pytest

import oracle
from lora_routing import references_by_adapter
from lora_support import check, f64, make


class _Host:
    """An array in the place of a result on the GPU."""

    def __init__(self, a):
        self.a = a

    def detach(self):
        return self

    cpu = double = detach

    def numpy(self):
        return self.a


@pytest.mark.parametrize("T,n,d_in,widths,r,kind", [(262144, 2048, 8, (8,), 8, "mixed"), (5000, 3, 16, (24, 8), 8, "runs")])
def test_a_missing_or_doubled_token_is_beyond_the_bound(T, n, d_in, widths, r, kind):
    c = make(T, n, d_in, widths, r, kind)
    ref = references_by_adapter(oracle, c)
    P = oracle.lora_fwd(*(f64(t) for t in (c.X, c.A, c.B, c.scale)), c.ids, f64(c.base), c.widths)[1]
    for name in ("dA", "dB"):
        check(name, _Host(ref[name][0]), ref[name])                     # the oracle's own result passes
    for token in np.flatnonzero(c.ids >= 0)[[0, T // 3, -1]]:
        a = c.ids[token]
        dy, x, s = f64(c.dY)[token], f64(c.X)[token], f64(c.scale)[a]
        first = slice(0, c.widths[0])
        q = s * (dy[first] @ f64(c.B)[a, first])
        for sign in (-1, 1):                                            # without the token, or with it twice
            for name, part in (("dB", s * np.outer(dy[first], P[token, :r])), ("dA", np.outer(q, x))):
                value = ref[name][0].copy()
                value[a, :part.shape[0]] += sign * part
                with pytest.raises(AssertionError, match=f"{name}: off by"):
                    check(name, _Host(value), ref[name])
