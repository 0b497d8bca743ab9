"""The adapters' gradients in tiles of 512, 1024 and 2048 tokens (tests/test_lora_plan.py checks the length of every
shape): several, partial and single tiles per adapter, ranks of every kernel, stacked parts, and the gradients without
dX, which take another launch."""
import pytest

import oracle
from gpu_support import say
from lora_routing import references_by_adapter, routed
from lora_support import backward, check, forward, plan_of, space

pytestmark = pytest.mark.gpu

LENGTHS = [  # tokens per adapter, n, d_in, widths, r, tokens without one, length of a gradient tile
    ((600,), 1, 4096, (22008,), 16, 0, 512),
    ((513, 510, 1), 5, 22008, (3000, 1096), 24, 0, 512),
    ((1000,), 1, 14000, (7000, 2504, 2496), 48, 24, 512),        # 144 stacked ranks
    ((1025, 900), 3, 2056, (24008,), 64, 40, 1024),
    ((1024, 33, 512), 3, 20008, (3080, 3096), 32, 5, 1024),
    ((2049, 40), 3, 4096, (21640,), 16, 11, 2048),
    ((31, 2050, 2047), 4, 25608, (1032,), 64, 0, 2048),
    ((4097,), 1, 9000, (8200,), 40, 0, 2048),
]


@pytest.mark.parametrize("counts,n,d_in,widths,r,none,length", LENGTHS)
def test_gradient_tiles(counts, n, d_in, widths, r, none, length):
    import paper_2609_33977_amd as gm
    import torch
    say(f"adapters: {counts} tokens and {none} without, {d_in} -> {widths}, r={r}, tiles of {length}")
    c = routed(counts, n, d_in, widths, r, none)
    Y, P = forward(gm, c)
    ref = references_by_adapter(oracle, c, P)
    dX, dA, dB = backward(gm, c, P)
    for name, got in (("Y", Y), ("P", P), ("dX", dX), ("dA", dA), ("dB", dB)):
        check(name, got, ref[name])
    alone = torch.full_like(dA, 3.0), torch.full_like(dB, 3.0)
    gm.gm_lora_bwd(c.dY.cuda(), c.X.cuda(), c.A.cuda(), c.B.cuda(), c.scale.cuda(), plan_of(gm, c.ids, n), P, None, None, *alone,
                   space(gm, gm.GM_OP_BWD, c), widths=widths)
    torch.cuda.synchronize()
    assert torch.equal(alone[0], dA) and torch.equal(alone[1], dB)
