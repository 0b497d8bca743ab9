"""Blocks of the adapters' Y and dX that are wider than the columns whose weights LDS holds, so that weights are loaded
anew in the middle of a block (tests/test_lora_plan.py checks the width of every shape): tiles of up to 16, up to 32 and
64 tokens, whose waves share the columns differently, last blocks that are not full, and dX with and without the
gradients, which are different launches."""
import pytest

import oracle
from gpu_support import say
from lora_routing import references_by_adapter, routed
from lora_support import backward, check, forward, plan_of, space

pytestmark = pytest.mark.gpu

TILES = (5, 16, 17, 32, 33, 70)   # tokens of the first adapters: tiles of up to 16, up to 32 and up to 64

WIDE = [  # d_in, widths, r, columns per block of the forward and of dX
    (24888, (12936,), 16, 1024, 1024),
    (25240, (12600, 984), 32, 1024, 1024),      # 64 stacked ranks
    (64, (600, 13000), 24, 1024, 256),
    (24600, (64,), 32, 256, 1024),
    (13064, (8200,), 64, 512, 512),
    (24936, (10200,), 64, 1024, 1024),
    (13064, (4200, 1032), 128, 512, 256),      # 256 stacked ranks: dX in rounds
    (13000, (3592,), 96, 1024, 512),
    (24712, (5000,), 72, 1024, 1024),
]


@pytest.mark.parametrize("d_in,widths,r,fwd,dx", WIDE)
def test_weights_loaded_anew_within_a_block(d_in, widths, r, fwd, dx):
    import paper_2609_33977_amd as gm
    import torch
    say(f"adapters: {TILES} tokens, {d_in} -> {widths}, r={r}, blocks of {fwd} columns (dX: {dx})")
    c = routed(TILES, 40, d_in, widths, r, none=3)
    Y, P = forward(gm, c)
    ref = references_by_adapter(oracle, c, P)
    dX, dA, dB = backward(gm, c, P)
    for name, got in (("Y", Y), ("P", P), ("dX", dX), ("dA", dA), ("dB", dB)):
        check(name, got, ref[name])
    alone = c.dXb.cuda()                        # in place, by itself
    gm.gm_lora_bwd(c.dY.cuda(), c.X.cuda(), c.A.cuda(), c.B.cuda(), c.scale.cuda(), plan_of(gm, c.ids, c.n), None, alone, alone,
                   ws=space(gm, gm.GM_OP_BWD, c), widths=widths)
    in_place, none = c.base.cuda(), plan_of(gm, c.ids, c.n)
    gm.gm_lora_fwd(c.X.cuda(), c.A.cuda(), c.B.cuda(), c.scale.cuda(), none, in_place, in_place, None, space(gm, gm.GM_OP_FWD, c),
                   widths=widths)
    torch.cuda.synchronize()
    assert torch.equal(alone, dX) and torch.equal(in_place, Y)
