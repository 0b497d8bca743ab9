"""The adapters' gradients against bounds by each adapter's own tokens, at every parity size and at the largest batch."""
import pytest

import oracle
from gpu_support import say
from lora_routing import references_by_adapter
from lora_support import backward, check, forward, make
from test_gpu_lora import SIZES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n,d_in,widths,r,kind", SIZES + [(262144, 2048, 8, (8,), 8, "mixed"), (262144, 1, 8, (16, 8), 8, "all"),
                                                            (262080, 2, 16, (8,), 16, "runs")])
def test_gradients(T, n, d_in, widths, r, kind):
    import paper_2609_33977_amd as gm
    say(f"adapters: T={T} n={n} d_in={d_in} widths={widths} r={r} routing {kind}")
    c = make(T, n, d_in, widths, r, kind)
    _, P = forward(gm, c)
    ref = references_by_adapter(oracle, c, P)
    for name, got in zip(("dX", "dA", "dB"), backward(gm, c, P)):
        check(name, got, ref[name])
