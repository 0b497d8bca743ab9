"""What calls may share: two captured graphs one plan and one workspace, calls on two streams one plan, a list without values."""
import pytest

from gpu_support import say
from lora_support import backward, forward, make, plan_of, space

pytestmark = pytest.mark.gpu


def _buffers(c):
    import torch
    return ([t.cuda() for t in (c.X, c.A, c.B, c.scale, c.base, c.dY, c.dXb)],
            [torch.empty(c.T, c.d_out, dtype=torch.bfloat16, device="cuda"), torch.empty(c.T, c.R, device="cuda"),
             torch.empty(c.T, c.d_in, dtype=torch.bfloat16, device="cuda"), torch.empty(c.A.shape, device="cuda"),
             torch.empty(c.B.shape, device="cuda")])


def _run(gm, c, data, out, plan, ws, stream=None):
    X, A, B, scale, base, dY, dXb = data
    gm.gm_lora_fwd(X, A, B, scale, plan, base, out[0], out[1], ws, widths=c.widths, stream=stream)
    gm.gm_lora_bwd(dY, X, A, B, scale, plan, out[1], dXb, *out[2:], ws, widths=c.widths, stream=stream)


def test_two_graphs_share_a_plan_and_a_workspace():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: graphs of two linears over one plan and one workspace, replayed in turn")
    cases = [make(150, 3, 264, (72, 64), 16, "mixed", seed=3), make(150, 3, 520, (648,), 64, "mixed", seed=3)]
    ids = torch.from_numpy(cases[0].ids).cuda()
    plan = torch.empty(gm.gm_lora_plan_size(150, 3), dtype=torch.uint8, device="cuda")
    ws = max((space(gm, op, c) for c in cases for op in (gm.GM_OP_FWD, gm.GM_OP_BWD)), key=lambda t: t.numel())
    held = [_buffers(c) for c in cases]
    gm.gm_lora_plan(ids, 3, plan)
    for c, (data, out) in zip(cases, held):
        _run(gm, c, data, out, plan, ws)
    torch.cuda.synchronize()
    graphs = []
    for c, (data, out) in zip(cases, held):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            _run(gm, c, data, out, plan, ws)
    for i in range(6):
        new = make(150, 3, 264, (72,), 16, ("runs", "mixed", "bad")[i % 3], seed=30 + i).ids    # the plan is made anew between replays
        ids.copy_(torch.from_numpy(new))
        gm.gm_lora_plan(ids, 3, plan)
        k = i % 2
        graphs[k].replay()
        graphs[1 - k].replay()
        torch.cuda.synchronize()
        for c, (_, out) in zip(cases, held):
            c.ids[:] = new
            Y, P = forward(gm, c)
            assert all(torch.equal(a, b) for a, b in zip(out, (Y, P, *backward(gm, c, P))))


def test_two_streams_share_a_plan():
    import paper_2609_33977_amd as gm
    import torch
    say("adapters: two linears on two streams over one plan")
    cases = [make(700, 4, 1032, (520,), 32, "mixed", seed=3), make(700, 4, 264, (1032, 136), 16, "mixed", seed=3)]
    want = []
    for c in cases:
        Y, P = forward(gm, c)
        want.append((Y, P, *backward(gm, c, P)))
    plan = plan_of(gm, cases[0].ids, 4)
    held = [_buffers(c) for c in cases]
    ws = [max((space(gm, op, c) for op in (gm.GM_OP_FWD, gm.GM_OP_BWD)), key=lambda t: t.numel()) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, (data, out), w, s in zip(cases, held, ws, streams):
            _run(gm, c, data, out, plan, w, stream=s)
    torch.cuda.synchronize()
    for (_, out), ref in zip(held, want):
        assert all(torch.equal(a, b) for a, b in zip(out, ref))


def test_a_list_without_values():
    import paper_2609_33977_amd as gm
    import torch
    from test_gpu_optim_lists import HYPER, _list, _norm
    say("lists of empty tensors only")
    for n in (1, 60):
        g, p, m, v = ([torch.empty(0, device="cuda") for _ in range(n)] for _ in range(4))
        lst = _list(gm, g, p=p, m=m, v=v)
        norm, coef = _norm(gm, lst, 1.0)
        assert float(norm) == 0.0 and float(coef) == 1.0
        gm.gm_adamw_list(lst, coef=coef, **HYPER)
        torch.cuda.synchronize()
