"""GPU parity of the low-rank adapters with the fp64 oracle: sizes around every tile, ranks, stacked parts, routings
(none, out of range, unused adapters, one adapter, runs), strides and aliasing, values that are not finite in other
tokens and adapters, order and determinism, streams, graphs, large offsets.  Bounds: tests/lora_support.py."""
import numpy as np
import pytest

import oracle
from gpu_support import say
from lora_support import backward, check, f64, forward, ids_of, make, plan_of, references, space

pytestmark = pytest.mark.gpu


def _both(c):
    import paper_2609_33977_amd as gm
    Y, P = forward(gm, c)
    ref = references(oracle, c, P)
    check("Y", Y, ref["Y"])
    check("P", P, ref["P"])
    dX, dA, dB = backward(gm, c, P)
    for name, got in (("dX", dX), ("dA", dA), ("dB", dB)):
        check(name, got, ref[name])
    return Y, P, dX, dA, dB


SIZES = [  # T, n, d_in, widths, r, routing
    (1, 1, 8, (8,), 8, "all"), (1, 3, 520, (264,), 16, "mixed"), (2, 2, 64, (40, 8), 8, "mixed"),
    (15, 4, 504, (72,), 24, "mixed"), (16, 1, 512, (512,), 16, "all"), (17, 1, 528, (520,), 16, "all"),
    (33, 2, 1032, (136, 24, 8), 16, "runs"), (63, 1, 128, (128,), 32, "all"), (64, 1, 136, (120,), 40, "all"),
    (65, 1, 1096, (264,), 48, "all"), (130, 70, 256, (64, 64), 16, "mixed"), (200, 3, 2056, (648,), 64, "runs"),
    (257, 1, 128, (256,), 72, "all"), (300, 5, 640, (40, 40, 40, 40), 128, "bad"), (513, 2, 72, (1032,), 16, "runs"),
    (600, 2048, 64, (32,), 8, "mixed"), (1000, 7, 264, (200, 56), 56, "bad"), (4100, 3, 40, (24,), 8, "runs"),
    (5000, 1, 136, (264,), 16, "all"), (12, 2, 24, (16,), 8, "none"),
    (20000, 1024, 16, (8,), 8, "mixed"), (9000, 1025, 8, (24,), 8, "bad"),
]


@pytest.mark.parametrize("T,n,d_in,widths,r,kind", SIZES)
def test_parity(T, n, d_in, widths, r, kind):
    say(f"adapters: T={T} n={n} d_in={d_in} widths={widths} r={r} routing {kind}")
    _both(make(T, n, d_in, widths, r, kind))


@pytest.mark.parametrize("widths", [(584, 112, 176, 144), (520, 128, 136), (2048, 256, 512, 264), (8, 1100 * 8)])
@pytest.mark.parametrize("r", [16, 32, 64])
def test_parts_much_narrower_than_the_widest(widths, r):
    # 70 tokens of one adapter: a tile of 64 and one of 6, whose narrow parts leave some of the contraction's splits empty
    say(f"adapters: T=70, widths={widths}, r={r}")
    _both(make(70, 1, 64, widths, r, "all"))


def test_the_largest_batch():
    say("adapters: 262144 tokens of 2048 adapters")
    _both(make(262144, 2048, 8, (8,), 8, "mixed"))


def test_llama2_7b_projections():
    say("adapters: T=96, q|k|v 4096 -> 3 x 4096, r=16; T=70, 11008 -> 4096, r=64")
    _both(make(96, 6, 4096, (4096, 4096, 4096), 16, "mixed"))
    _both(make(70, 2, 11008, (4096,), 64, "runs"))


def test_gradients_against_differences():
    # sum(dY Y) is linear in A and in B: a step D changes it by sum(dA D).  base = 0, so Y's rounding is 2^-8 of the
    # update itself; it enters twice, with the fp32 products' error far below it.
    import dataclasses

    import paper_2609_33977_amd as gm
    import torch
    c = make(150, 2, 320, (136,), 16, "runs", seed=5)
    c = dataclasses.replace(c, base=torch.zeros_like(c.base))
    _, P = forward(gm, c)
    _, dA, dB = backward(gm, c, P)
    g = torch.Generator().manual_seed(11)
    for name, grad in (("A", dA), ("B", dB)):
        w = getattr(c, name)
        D = (torch.randn(w.shape, generator=g) * 0.5).to(torch.bfloat16)
        hi, lo = ((w.float() + s * D.float()).to(torch.bfloat16) for s in (1, -1))
        Yh, Yl = (f64(forward(gm, dataclasses.replace(c, **{name: v}))[0]) for v in (hi, lo))
        dY = f64(c.dY)
        change = float(np.sum(dY * (Yh - Yl)))
        want = float(np.sum(f64(grad) * (f64(hi) - f64(lo))))
        bound = 2.0 ** -7.9 * float(np.sum(np.abs(dY) * (np.abs(Yh) + np.abs(Yl))))
        say(f"difference along {name}: {change:.4f}, by the gradient {want:.4f}, bound {bound:.4f}")
        assert abs(change - want) <= bound


def test_columns_of_wider_buffers_and_in_place():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: strided X, base, Y, dY, dX; guards; in place")
    c = make(77, 3, 264, (72, 40), 16, "mixed")
    Y, P = forward(gm, c)
    dX, dA, dB = backward(gm, c, P)
    plan, guard = plan_of(gm, c.ids, c.n), 5.0

    def wide(t, left, right):
        w = torch.full((t.shape[0] + 2, left + t.shape[1] + right), guard, dtype=t.dtype, device="cuda")
        v = w[1:-1, left:left + t.shape[1]]
        v.copy_(t)
        return w, v

    def guards_kept(w, v, left):
        w = w.clone()
        w[1:-1, left:left + v.shape[1]] = guard
        return bool((w == guard).all())

    A, B, scale = c.A.cuda(), c.B.cuda(), c.scale.cuda()
    _, X = wide(c.X, 8, 24)
    _, base = wide(c.base, 16, 8)
    wy, y = wide(torch.zeros_like(c.base), 24, 16)
    P2 = torch.empty_like(P)
    gm.gm_lora_fwd(X, A, B, scale, plan, base, y, P2, space(gm, gm.GM_OP_FWD, c), widths=c.widths)
    wb, yb = wide(c.base, 40, 8)
    gm.gm_lora_fwd(X, A, B, scale, plan, yb, yb, None, space(gm, gm.GM_OP_FWD, c), widths=c.widths)
    torch.cuda.synchronize()
    assert torch.equal(y, Y) and torch.equal(yb, Y) and torch.equal(P2, P)
    assert guards_kept(wy, y, 24) and guards_kept(wb, yb, 40)
    _, dY = wide(c.dY, 8, 8)
    wx, dx = wide(c.dXb, 8, 16)
    dA2, dB2 = torch.empty_like(dA), torch.empty_like(dB)
    gm.gm_lora_bwd(dY, X, A, B, scale, plan, P, dx, dx, dA2, dB2, space(gm, gm.GM_OP_BWD, c), widths=c.widths)
    torch.cuda.synchronize()
    assert torch.equal(dx, dX) and torch.equal(dA2, dA) and torch.equal(dB2, dB) and guards_kept(wx, dx, 8)


def test_each_output_alone():
    import paper_2609_33977_amd as gm
    import torch
    c = make(300, 4, 136, (72, 72), 24, "mixed")
    _, P = forward(gm, c)
    dX, dA, dB = backward(gm, c, P)
    plan, ws = plan_of(gm, c.ids, c.n), space(gm, gm.GM_OP_BWD, c)
    args = [t.cuda() for t in (c.dY, c.X, c.A, c.B, c.scale)]
    for k in range(1, 8):
        out = [torch.empty_like(t) if k >> i & 1 else None for i, t in enumerate((dX, dA, dB))]
        gm.gm_lora_bwd(*args, plan, P if out[2] is not None else None, c.dXb.cuda() if out[0] is not None else None, *out, ws,
                       widths=c.widths)
        torch.cuda.synchronize()
        for got, want in zip(out, (dX, dA, dB)):
            assert got is None or torch.equal(got, want)
    gm.gm_lora_bwd(*args, plan, None, ws=ws, widths=c.widths)


def test_rows_without_an_adapter_and_unused_adapters():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: NaN and infinities in other tokens, in tokens without an adapter and in adapters that no token has")
    c = make(90, 6, 264, (136,), 16, "mixed", seed=9)
    c.ids[c.ids == 4] = -1                      # adapter 4 is unused
    Y, P = forward(gm, c)
    dX, dA, dB = backward(gm, c, P)
    none = torch.from_numpy(c.ids < 0)
    assert int(none.sum()) > 0
    assert torch.equal(Y.cpu()[none], c.base[none]) and torch.equal(dX.cpu()[none], c.dXb[none])
    assert not P.cpu()[none].any() and not dA[4].any() and not dB[4].any()
    sick = 2                                    # a token's adapter 2 is sick, and so are rows without one
    for bad in (float("nan"), float("inf")):
        X, dY, A, B, scale = (t.clone() for t in (c.X, c.dY, c.A, c.B, c.scale))
        for t in (X, dY):
            t[none] = bad
            t[int(np.flatnonzero(c.ids == sick)[0])] = bad
        for t in (A, B, scale):
            t[4] = bad
        A[sick, 3, 5] = bad
        import dataclasses
        s = dataclasses.replace(c, X=X, dY=dY, A=A, B=B, scale=scale)
        Y2, P2 = forward(gm, s)
        dX2, dA2, dB2 = backward(gm, s, P2)
        well = torch.from_numpy(c.ids != sick)
        others = [a for a in range(c.n) if a != sick]
        assert torch.equal(Y2.cpu()[well], Y.cpu()[well]) and torch.equal(P2.cpu()[well], P.cpu()[well])
        assert torch.equal(dX2.cpu()[well], dX.cpu()[well])
        assert torch.equal(dA2[others], dA[others]) and torch.equal(dB2[others], dB[others])
        assert not torch.isfinite(Y2.cpu()[~well].float()).all()


def test_order_of_the_batch_and_repeats():
    import dataclasses

    import paper_2609_33977_amd as gm
    import torch
    c = make(700, 5, 520, (264,), 16, "mixed", seed=4)
    first = [*forward(gm, c), *backward(gm, c, forward(gm, c)[1])]
    again = [*forward(gm, c), *backward(gm, c, first[1])]
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    p = torch.randperm(c.T, generator=torch.Generator().manual_seed(2))
    s = dataclasses.replace(c, ids=c.ids[p.numpy()], X=c.X[p], base=c.base[p], dY=c.dY[p], dXb=c.dXb[p])
    Y, P = forward(gm, s)
    ref = references(oracle, s, P)
    for name, got in zip(("Y", "P", "dX", "dA", "dB"), (Y, P, *backward(gm, s, P))):
        check(name, got, ref[name])


def test_one_plan_for_linears_of_other_sizes():
    import paper_2609_33977_amd as gm
    import torch
    ids = ids_of("mixed", 123, 4, 8)
    plan = plan_of(gm, ids, 4)
    for d_in, widths, r in ((64, (64,), 8), (520, (24, 40), 32), (1032, (136,), 64)):
        c = make(123, 4, d_in, widths, r, "mixed", seed=8)
        assert np.array_equal(c.ids, ids)
        Y, P = forward(gm, c, plan)
        ref = references(oracle, c, P)
        check("Y", Y, ref["Y"])
        for name, got in zip(("dX", "dA", "dB"), backward(gm, c, P, plan)):
            check(name, got, ref[name])
    torch.cuda.synchronize()


def test_a_plan_for_other_sizes_writes_nothing():
    import paper_2609_33977_amd as gm
    import torch
    c = make(100, 3, 64, (64,), 16, "mixed")
    other = plan_of(gm, ids_of("mixed", 200, 3, 1), 3)    # larger, and made for 200 tokens
    Y, P = forward(gm, c, other)
    assert bool((Y == 3.0).all()) and bool((P == 3.0).all())
    for t in backward(gm, c, torch.zeros(c.T, c.R), other):
        assert bool((t == 3.0).all())


def test_streams_and_workspaces():
    import paper_2609_33977_amd as gm
    import torch
    cases = [make(90 + 7 * i, 3, 264, (136,), 16, "mixed", seed=i) for i in range(3)]
    want = [forward(gm, c) for c in cases]
    data = [[t.cuda() for t in (c.X, c.A, c.B, c.scale, c.base)] for c in cases]
    ids = [torch.from_numpy(c.ids).cuda() for c in cases]
    ws = [space(gm, gm.GM_OP_FWD, c) for c in cases]
    plans = [torch.empty(gm.gm_lora_plan_size(c.T, c.n), dtype=torch.uint8, device="cuda") for c in cases]
    outs = [(torch.empty_like(Y), torch.empty_like(P)) for Y, P in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for c, (X, A, B, scale, base), i, w, plan, (Y, P), s in zip(cases, data, ids, ws, plans, outs, streams):
        gm.gm_lora_plan(i, c.n, plan, stream=s)
        gm.gm_lora_fwd(X, A, B, scale, plan, base, Y, P, w, widths=c.widths, stream=s)
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_captured_and_replayed():
    # plan, forward, backward, norm and step of one captured graph, replayed with new inputs, eager work between
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: graph of a whole step, four replays")
    c = make(140, 3, 264, (72, 64), 16, "mixed")
    buf = {k: getattr(c, k).cuda() for k in ("X", "A", "B", "scale", "base", "dY", "dXb")}
    ids = torch.from_numpy(c.ids).cuda()
    plan = torch.empty(gm.gm_lora_plan_size(c.T, c.n), dtype=torch.uint8, device="cuda")
    wf, wb = space(gm, gm.GM_OP_FWD, c), space(gm, gm.GM_OP_BWD, c)
    out = [torch.empty(c.T, c.d_out, dtype=torch.bfloat16, device="cuda"), torch.empty(c.T, c.R, device="cuda"),
           torch.empty(c.T, c.d_in, dtype=torch.bfloat16, device="cuda"), torch.empty(c.A.shape, device="cuda"),
           torch.empty(c.B.shape, device="cuda")]
    lst = torch.empty(gm.gm_tensor_list_size([c.A.numel(), c.B.numel()]), dtype=torch.uint8, device="cuda")
    gm.gm_tensor_list(out[3:], lst)
    norm, coef = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    nws = torch.empty(gm.GM_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def step():
        gm.gm_lora_plan(ids, c.n, plan)
        gm.gm_lora_fwd(buf["X"], buf["A"], buf["B"], buf["scale"], plan, buf["base"], out[0], out[1], wf, widths=c.widths)
        gm.gm_lora_bwd(buf["dY"], buf["X"], buf["A"], buf["B"], buf["scale"], plan, out[1], buf["dXb"], *out[2:], wb,
                       widths=c.widths)
        gm.gm_grad_norm(lst, 1.0, norm, coef, nws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        s = make(140, 3, 264, (72, 64), 16, ("runs", "mixed", "none", "bad")[i], seed=20 + i)
        for k in buf:
            buf[k].copy_(getattr(s, k))
        ids.copy_(torch.from_numpy(s.ids))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, norm, coef)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out, norm, coef)))
        ref = references(oracle, s, got[1])
        for name, t in zip(("Y", "P", "dX", "dA", "dB"), got):
            check(name, t, ref[name])


def test_offsets_past_32_bits():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: a pool of 4.6 GB and rows 4.4 GB apart")
    n, r, d_in, T, ld = 1100, 64, 32768, 2112, (1 << 20) + 8
    A = torch.zeros(n, r, d_in, dtype=torch.bfloat16, device="cuda")
    c = make(T, 2, d_in, (64,), r, "runs", seed=3)
    c.ids[:] = np.where(np.arange(T) < 5, n - 1, -1)
    c.ids[-3:] = 0
    wide = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    X = wide.as_strided((T, d_in), (ld, 1))
    X.copy_(c.X)
    A[0].copy_(c.A[0]), A[n - 1].copy_(c.A[1])
    B = torch.zeros(n, 64, r, dtype=torch.bfloat16, device="cuda")
    B[0].copy_(c.B[0]), B[n - 1].copy_(c.B[1])
    scale = torch.ones(n, device="cuda")
    Y, P = torch.empty(T, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(T, r, device="cuda")
    plan = plan_of(gm, c.ids, n)
    ws = torch.empty(gm.gm_lora_workspace_size(gm.GM_OP_FWD, T, n, d_in, 64, r), dtype=torch.uint8, device="cuda")
    gm.gm_lora_fwd(X, A, B, scale, plan, c.base.cuda(), Y, P, ws)
    torch.cuda.synchronize()
    c.ids = np.where(c.ids == n - 1, 1, c.ids)
    c.scale = torch.ones(2)
    ref = references(oracle, c)
    check("Y", Y, ref["Y"])
    check("P", P, ref["P"])


def test_beside_the_masked_and_the_packed_linear():
    # as they are used together: the pruned linear's output is the base, in place; the masked backward's dX likewise;
    # then the norm over both gradients and the clipped step, whose bf16 copies the next forward reads
    import paper_2609_33977_amd as gm
    import torch
    import workloads
    from gpu_support import dev_bf16, dev_f32, workspace
    say("adapters beside the masked and packed linears, and one clipped step on them")
    T, d_in, d_out, g, r, n = 96, 512, 512, 128, 16, 2
    case = workloads.make_linear_case((77, 1), T, d_in, d_out, g, None)
    X, W, dY, mask = dev_bf16(case.X), dev_bf16(case.W), dev_bf16(case.dY), dev_f32(case.mask)
    G, cap = d_in // g, d_out * (d_in // g)
    Wp, chunk = torch.empty(cap, g, dtype=torch.bfloat16, device="cuda"), torch.empty(cap, dtype=torch.int32, device="cuda")
    sc, rowptr = torch.empty(cap, device="cuda"), torch.empty(d_out + 1, dtype=torch.int32, device="cuda")
    gm.gm_pack_rows(W, mask, g, cap, Wp, chunk, sc, rowptr)
    Ym, Yp = (torch.empty(T, d_out, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gm.gm_masked_linear_fwd(X, W, mask, g, Ym)
    gm.gm_packed_linear_fwd(X, Wp, chunk, sc, rowptr, d_out, g, Yp)
    c = make(T, n, d_in, (d_out,), r, "runs", seed=6)
    plan = plan_of(gm, c.ids, n)
    A, B, scale = c.A.cuda(), c.B.cuda(), c.scale.cuda()
    P = torch.empty(T, r, device="cuda")
    bases = {"masked": Ym.clone(), "packed": Yp.clone()}
    for Y in (Ym, Yp):
        gm.gm_lora_fwd(X, A, B, scale, plan, Y, Y, P, space(gm, gm.GM_OP_FWD, c))
    dX, dg = torch.empty(T, d_in, dtype=torch.bfloat16, device="cuda"), torch.empty(d_out, G, device="cuda")
    gm.gm_masked_linear_bwd(dY, X, W, mask, g, dX, dg, workspace(gm.gm_workspace_size(gm.GM_OP_BWD, T, d_in, d_out, g)))
    torch.cuda.synchronize()
    dX_base = dX.clone()
    grads = [torch.empty(c.A.shape, device="cuda"), torch.empty(c.B.shape, device="cuda")]
    gm.gm_lora_bwd(dY, X, A, B, scale, plan, P, dX, dX, *grads, space(gm, gm.GM_OP_BWD, c))
    p = [A.float(), B.float()]
    m, v = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
    copies = [A, B]                                        # the working copies are the kernels' own inputs
    lst = torch.empty(gm.gm_tensor_list_size([t.numel() for t in p]), dtype=torch.uint8, device="cuda")
    gm.gm_tensor_list(grads, lst, p=p, m=m, v=v, p16=copies)
    norm, coef = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    nws = torch.empty(gm.GM_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    before = [t.clone() for t in copies]
    gm.gm_grad_norm(lst, 0.5, norm, coef, nws)
    gm.gm_adamw_list(lst, 1e-3, 0.9, 0.999, 1e-8, 0.05, 1, coef)
    torch.cuda.synchronize()
    c.X, c.dY, c.dXb = X.cpu(), dY.cpu(), dX_base.cpu()
    for name, Y in (("masked", Ym), ("packed", Yp)):
        c.base = bases[name].cpu()
        ref = references(oracle, c, P)
        check(f"Y ({name})", Y, ref["Y"])
    check("dX", dX, ref["dX"])
    check("dA", grads[0], ref["dA"])
    check("dB", grads[1], ref["dB"])
    want, k = oracle.grad_norm([f64(t) for t in grads], 0.5)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want and abs(float(coef) - k) <= 2.0 ** -23 * k and k < 1
    for w32, w16, old in zip(p, copies, before):
        assert torch.equal(w16, w32.to(torch.bfloat16)) and not torch.equal(w16, old)
