"""The adapters' backward past 32 bits: a pool whose A and dA, B and dB hold more than 2^31 values each, partial sums of
gradient tiles beyond 2^31 values, and rows of dY, X and dX gigabytes apart."""
import numpy as np
import pytest

import oracle
from gpu_support import say
from lora_routing import references_by_adapter, routed
from lora_support import check, f64, plan_of

pytestmark = pytest.mark.gpu


def test_gradients_of_a_pool_past_32_bits():
    import paper_2609_33977_amd as gm
    import torch
    # adapters 0 and n - 1 of a pool of zeros; the last has two gradient tiles, whose partial sums come after the others'
    n, r, d = 1100, 64, 32768
    last = 2100
    say(f"adapters: gradients of {n} adapters, {r} ranks, {d} columns each way ({n * r * d * 4 / 1e9:.1f} GB)")
    c = routed((3, last), 2, d, (d,), r)
    T = 3 + last + n - 2
    ids = np.concatenate([np.where(c.ids == 1, n - 1, 0), np.arange(1, n - 1)]).astype(np.int32)   # one token for each other

    def rows(t):
        return torch.cat([t, t[:1].expand(n - 2, d)]).cuda()

    A, B = (torch.zeros(n, *s, dtype=torch.bfloat16, device="cuda") for s in ((r, d), (d, r)))
    for w, own in ((A, c.A), (B, c.B)):
        w[0].copy_(own[0]), w[n - 1].copy_(own[1])
    scale = torch.ones(n, device="cuda")
    scale[0], scale[n - 1] = c.scale[0], c.scale[1]
    plan = plan_of(gm, ids, n)
    X, dY, base, dXb = (rows(t) for t in (c.X, c.dY, c.base, c.dXb))
    ws = torch.empty(max(gm.gm_lora_workspace_size(op, T, n, d, d, r) for op in (gm.GM_OP_FWD, gm.GM_OP_BWD)), dtype=torch.uint8,
                     device="cuda")
    P = torch.empty(T, r, device="cuda")
    gm.gm_lora_fwd(X, A, B, scale, plan, base, base, P, ws)
    dX = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    dA, dB = (torch.full(w.shape, 3.0, device="cuda") for w in (A, B))
    gm.gm_lora_bwd(dY, X, A, B, scale, plan, P, dXb, dX, dA, dB, ws)
    torch.cuda.synchronize()
    own = 3 + last
    ref = references_by_adapter(oracle, c, P[:own])
    check("Y", base[:own], ref["Y"])
    check("dX", dX[:own], ref["dX"])
    for name, grad in (("dA", dA), ("dB", dB)):
        check(name, grad[[0, n - 1]], ref[name])
        for k in range(1, n - 1, 100):                                  # a slice at a time
            assert not grad[k:min(k + 100, n - 1)].any()
    assert torch.equal(dX[own:], dXb[own:])


def test_rows_past_32_bits():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: rows of X, dY and dX 2 MB apart, 4.4 GB each")
    T, ld = 2112, (1 << 20) + 8
    c = routed((2000, 100), 3, 520, (264,), 16, none=12)

    def wide(t):
        w = torch.zeros(T * ld, dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
        return w.copy_(t)

    plan = plan_of(gm, c.ids, c.n)
    A, B, scale = c.A.cuda(), c.B.cuda(), c.scale.cuda()
    X, dY, dX = wide(c.X), wide(c.dY), wide(c.dXb)
    ws = torch.empty(max(gm.gm_lora_workspace_size(op, T, c.n, c.d_in, c.widths, c.r) for op in (gm.GM_OP_FWD, gm.GM_OP_BWD)),
                     dtype=torch.uint8, device="cuda")
    Y, P = torch.empty(T, c.d_out, dtype=torch.bfloat16, device="cuda"), torch.empty(T, c.R, device="cuda")
    gm.gm_lora_fwd(X, A, B, scale, plan, c.base.cuda(), Y, P, ws)
    dA, dB = torch.empty(A.shape, device="cuda"), torch.empty(B.shape, device="cuda")
    gm.gm_lora_bwd(dY, X, A, B, scale, plan, P, dX, dX, dA, dB, ws)
    torch.cuda.synchronize()
    assert np.array_equal(f64(X), f64(c.X)) and np.array_equal(f64(dY), f64(c.dY))
    ref = references_by_adapter(oracle, c, P)
    for name, got in (("Y", Y), ("dX", dX), ("dA", dA), ("dB", dB)):
        check(name, got, ref[name])
