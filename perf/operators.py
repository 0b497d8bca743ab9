"""Operators of tuning and serving low-rank adapters on a pruned model, and of clipped optimiser steps: cases and plain forms.

A pruned linear keeps its frozen weight; what is lost is won back by a low-rank adapter beside it, and one pruned model
serves the adapters of many requests at once.  For a token t with adapter a (none where its id is outside 0 .. n - 1):

  P[t] = X[t] A_a^T                               [r]
  Y[t] = base[t] + scale_a P[t] B_a^T             base: the output of the masked or packed linear
  Q[t] = scale_a dY[t] B_a                        [r]
  dX[t] = base[t] + Q[t] A_a                      base: the dX of the masked linear
  dA_a = sum over a's tokens of Q[t]^T X[t],  dB_a = scale_a sum over a's tokens of dY[t]^T P[t]

and over all gradients g of a step

  norm = sqrt(sum g^2),  coef = min(1, max_norm / norm)

with which AdamW then updates every tensor (decoupled decay, bias-corrected moments) and its bf16 working copy.

Kinds of cases:
  serve    the routing of one batch, then the adapters of a decoder layer's seven projections, those that read one
           input stacked side by side (q|k|v, gate|up), as the packed linear has them
  project  the routing and the adapter of one projection, its P kept for the backward
  grad     the routing and the backward of one projection
  norm     the norm over many tensors and the clipping coefficient
  step     the norm and the clipped AdamW step over many tensors, on copies of parameters and moments
  tune     one projection's whole step: routing, forward, backward, norm, AdamW on the adapters' fp32 masters
"""
import math

import torch

own = False

# (d_model, d_ff) of the two models whose projections the workloads use.
MODELS = {"7b": (4096, 11008), "13b": (5120, 13824)}
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.05, 7


def listed():
    return [
        # One generated token of one request through a decoder layer: launches count.
        {"name": "serve_7b_t1", "kind": "serve", "model": "7b", "T": 1, "n": 8, "r": 16, "none": 0.0, "runs": False},
        # A decode batch, one token a request, adapters drawn from a pool, some requests without one.
        {"name": "serve_13b_t64", "kind": "serve", "model": "13b", "T": 64, "n": 32, "r": 16, "none": 0.1, "runs": False},
        # A large decode batch of high-rank adapters, an odd number of tokens.
        {"name": "serve_7b_t203_r64", "kind": "serve", "model": "7b", "T": 203, "n": 40, "r": 64, "none": 0.1, "runs": False},
        # Prompts of a dozen requests packed into one batch, each with its own adapter.
        {"name": "project_prompts_t4099", "kind": "project", "T": 4099, "d_in": 4096, "d_out": 11008, "parts": 1, "n": 12, "r": 16, "none": 0.05, "runs": True},
        # Training forward of the widest input at 4 x 2048 tokens, one adapter of high rank.
        {"name": "project_down_t8192_r64", "kind": "project", "T": 8192, "d_in": 11008, "d_out": 4096, "parts": 1, "n": 1, "r": 64, "none": 0.0, "runs": True},
        # Training backward of the stacked q|k|v projections at the paper's batch of 1 x 2048 tokens.
        {"name": "grad_qkv_t2048", "kind": "grad", "T": 2048, "d_in": 4096, "d_out": 4096, "parts": 3, "n": 1, "r": 16, "none": 0.0, "runs": True},
        # Several tenants tuned in one batch; sizes that no tile divides, a rank that is no power of two.
        {"name": "grad_ragged_t1000", "kind": "grad", "T": 1000, "d_in": 2816, "d_out": 2056, "parts": 1, "n": 5, "r": 24, "none": 0.1, "runs": True},
        # Training backward of an MLP projection at 4 x 2048 tokens, high rank: the largest call.
        {"name": "grad_up_t8192_r64", "kind": "grad", "T": 8192, "d_in": 4096, "d_out": 11008, "parts": 1, "n": 1, "r": 64, "none": 0.0, "runs": True},
        # The gradients of one small module: two launches' latency.
        {"name": "norm_small", "kind": "norm", "tensors": 4, "most": 12352, "bf16": False},
        # Every adapter gradient of a 7B model at rank 16: 448 tensors, 40 M values.
        {"name": "norm_7b_r16", "kind": "norm", "tensors": 448, "most": 176128, "bf16": False},
        # The clipped step over the same tensors.
        {"name": "step_7b_r16", "kind": "step", "tensors": 448, "most": 176128},
        # One projection's adapter tuned for a step on 2 x 2048 tokens.
        {"name": "tune_attn_t4096", "kind": "tune", "T": 4096, "d_in": 4096, "d_out": 4096, "parts": 1, "n": 2, "r": 16, "none": 0.0, "runs": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["serve", "serve", "project", "project", "grad", "grad", "norm", "step", "tune"])
    if kind == "norm":
        return {"kind": kind, "tensors": _log(rng, 1, 448), "most": _log(rng, 500, 176128), "bf16": rng.random() < 0.3}
    if kind == "step":
        return {"kind": kind, "tensors": _log(rng, 1, 448), "most": _log(rng, 500, 176128)}
    case = {"kind": kind, "r": rng.choice([8, 16, 16, 24, 32, 48, 64]), "none": rng.choice([0.0, 0.1]), "runs": kind != "serve"}
    if kind == "serve":
        return case | {"model": rng.choice(["7b", "13b"]), "T": _log(rng, 1, 256), "n": _log(rng, 1, 40)}
    d_in, d_out, parts = 8 * _log(rng, 32, 1376), 8 * _log(rng, 32, 1376), rng.choice([1, 1, 2, 3])
    most = min(8192, 8192 * (4096 + 11008) // (d_in + parts * d_out))
    if kind == "tune":
        most = min(most, 4096)
    return case | {"T": _log(rng, 17, most), "d_in": d_in, "d_out": d_out, "parts": parts, "n": _log(rng, 1, 16)}


# ---------------------------------------------------------------- inputs

def _linears(model):
    """Per input of a decoder layer: (d_in, output widths of the projections that read it)."""
    d, f = MODELS[model]
    return [(d, [d, d, d]), (d, [d]), (d, [f, f]), (f, [d])]


def _groups(case):
    return _linears(case["model"]) if case["kind"] == "serve" else [(case["d_in"], [case["d_out"]] * case["parts"])]


def _sizes(case):
    """Element counts of a step's tensors: the largest first, then spread below it, odd ones among them."""
    gen = torch.Generator().manual_seed(17)
    low = max(1, case["most"] // 8)
    some = torch.randint(low, case["most"] + 1, (case["tensors"],), generator=gen)
    some[0] = case["most"]
    return [int(v) for v in some]


def _ids(case, seed):
    """Each token's adapter: runs of one request's tokens, or a request per token; -1 for none."""
    gen = torch.Generator().manual_seed(1000003 * seed + 29)
    T, n = case["T"], case["n"]
    if case["runs"]:
        cuts = torch.randint(0, T, (min(T, n + 2) - 1,), generator=gen)
        run = torch.zeros(T, dtype=torch.int64)
        run.index_add_(0, cuts, torch.ones_like(cuts))
        run = torch.cumsum(run, 0)
        ids = run % n
        ids[(run == 1) & (case["none"] > 0)] = -1
    else:
        ids = torch.randint(0, n, (T,), generator=gen)
        ids[torch.rand(T, generator=gen) < case["none"]] = -1
    return ids.to(torch.int32).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

    s = {"case": case}
    kind = case["kind"]
    if kind in ("norm", "step"):
        sizes = _sizes(case)
        total = sum(sizes)
        s["sizes"] = sizes
        s["g"] = normal(total, std=1e-3, dtype=torch.bfloat16 if case.get("bf16") else torch.float32)
        s["max_norm"] = 0.5e-3 * math.sqrt(total)
        if kind == "step":
            s["p"] = normal(total, std=0.02, dtype=torch.float32)
            s["m"] = normal(total, std=1e-3, dtype=torch.float32)
            s["v"] = 1e-6 * (0.25 + normal(total, dtype=torch.float32).square_())
            s["p_new"], s["m_new"], s["v_new"] = (torch.empty_like(s["p"]) for _ in range(3))
            s["p16"] = torch.empty(total, dtype=torch.bfloat16, device="cuda")
    else:
        s["ids"] = _ids(case, seed)
        T, n, r = case["T"], case["n"], case["r"]
        s["scale"] = 0.5 + 1.5 * torch.rand(n, generator=gen, device="cuda")
        groups = _groups(case)
        s["X"] = [normal(T, d_in) for d_in, _ in groups]
        s["base"] = [normal(T, sum(outs)) for _, outs in groups]
        s["Y"] = [torch.empty_like(b) for b in s["base"]]
        # Freshly initialised adapters start at B = 0; these are trained ones.
        s["A"] = [normal(n, len(outs) * r, d_in, std=1 / math.sqrt(d_in)) for d_in, outs in groups]
        s["B"] = [normal(n, sum(outs), r, std=0.3 / math.sqrt(r)) for _, outs in groups]
        s["widths"] = [outs for _, outs in groups]
        if kind in ("grad", "tune"):
            s["dY"] = normal(T, sum(s["widths"][0]), std=1e-2)
            s["dX_base"] = normal(T, case["d_in"], std=1e-2)
            s["dX"] = torch.empty_like(s["dX_base"])
            s["dA"], s["dB"] = (torch.empty(w.shape, device="cuda") for w in (s["A"][0], s["B"][0]))
        if kind == "project" or kind == "tune":
            s["P"] = torch.empty(T, r * case["parts"], device="cuda")
        if kind == "grad":  # kept from the forward
            s["P"] = torch.cat([_low(s["X"][0].float(), a, s["ids"]) for a in s["A"][0].split(r, 1)], dim=1)
        if kind == "tune":
            # fp32 masters whose bf16 copies the kernels read, both adapters' matrices in one buffer
            master = torch.cat([s["A"][0].float().flatten(), s["B"][0].float().flatten()])
            s["max_norm"] = 1e-3 * math.sqrt(master.numel())
            s["p"] = master + 1e-5 * normal(master.numel(), dtype=torch.float32) * master.abs()
            s["m"] = normal(master.numel(), std=1e-3, dtype=torch.float32)
            s["v"] = 1e-6 * (0.25 + normal(master.numel(), dtype=torch.float32).square_())
            s["p_new"], s["m_new"], s["v_new"] = (torch.empty_like(s["p"]) for _ in range(3))
            s["p16"] = torch.empty(master.numel(), dtype=torch.bfloat16, device="cuda")
    if kind in ("norm", "step", "tune"):
        s["norm"] = torch.empty(1, device="cuda")
        s["coef"] = torch.empty(1, device="cuda")
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program of the framework keeps: workspaces, and the list of the tensors that its optimiser steps."""
    import paper_2609_33977_amd as gm
    case, kind = s["case"], s["case"]["kind"]

    def space(nbytes):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")

    if kind not in ("norm", "step"):
        T, n, r = case["T"], case["n"], case["r"]
        s["plan"] = space(gm.gm_lora_plan_size(T, n))
        ops = [gm.GM_OP_FWD] * (kind != "grad") + [gm.GM_OP_BWD] * (kind in ("grad", "tune"))
        s["ws"] = space(max(gm.gm_lora_workspace_size(op, T, n, X.shape[1], widths, r)
                            for op in ops for X, widths in zip(s["X"], s["widths"])))
    if kind in ("norm", "step", "tune"):
        if kind == "tune":
            sizes, grads = [s["dA"].numel(), s["dB"].numel()], [s["dA"], s["dB"]]
        else:
            sizes, grads = s["sizes"], s["g"].split(s["sizes"])
        rest = {} if kind == "norm" else {k: s[f].split(sizes) for k, f in
                                          (("p", "p_new"), ("m", "m_new"), ("v", "v_new"), ("p16", "p16"))}
        s["list"] = space(gm.gm_tensor_list_size(sizes))
        gm.gm_tensor_list(grads, s["list"], **rest)
        s["norm_ws"] = space(gm.GM_GRAD_NORM_WORKSPACE_BYTES)


# ---------------------------------------------------------------- the plain form

def _chosen(ids, n, r):
    """[T, n r]: where token t's row of the stacked ranks belongs to its own adapter."""
    return (ids[:, None] == torch.arange(n, device=ids.device, dtype=ids.dtype)).repeat_interleave(r, dim=1)


def _wide(X, A, ids):
    """X A^T over all adapters' ranks side by side, zero outside the token's own: [T, n r]."""
    n, r, d_in = A.shape
    return torch.where(_chosen(ids, n, r), X @ A.float().reshape(n * r, d_in).t(), 0.0)


def _low(X, A, ids):
    n, r, _ = A.shape
    return _wide(X, A, ids).reshape(-1, n, r).sum(1)


def _stack(B):
    """[n, d_out, r] -> [n r, d_out] in 32 bits."""
    n, d_out, r = B.shape
    return B.float().transpose(1, 2).reshape(n * r, d_out)


def _forward(X, A, B, scale, ids, base):
    n, r, _ = A.shape
    P = _wide(X.float(), A, ids)
    return (base.float() + (P * scale.repeat_interleave(r)) @ _stack(B)).to(base.dtype), P


def _forwards(s, i):
    """Y and P of each part of stack i."""
    r, widths = s["case"]["r"], s["widths"][i]
    return [_forward(s["X"][i], a, b, s["scale"], s["ids"], c)
            for a, b, c in zip(s["A"][i].split(r, 1), s["B"][i].split(widths, 1), s["base"][i].split(widths, 1))]


def _backward(s, Ps):
    """Ps: for each part of the stack [T, n r], zero outside the token's own adapter."""
    n, r, widths = s["case"]["n"], s["case"]["r"], s["widths"][0]
    X, dYs = s["X"][0].float(), s["dY"].float().split(widths, 1)
    As = [a.float().reshape(n * r, -1) for a in s["A"][0].split(r, 1)]
    by_rank = s["scale"].repeat_interleave(r)
    Qs = [torch.where(_chosen(s["ids"], n, r), dY @ _stack(b).t(), 0.0) * by_rank
          for dY, b in zip(dYs, s["B"][0].split(widths, 1))]
    dX = (s["dX_base"].float() + sum(Q @ a for Q, a in zip(Qs, As))).to(s["dX_base"].dtype)
    dA = torch.cat([(Q.t() @ X).reshape(n, r, -1) for Q in Qs], dim=1)
    dB = torch.cat([((P * by_rank).t() @ dY).reshape(n, r, -1).transpose(1, 2) for P, dY in zip(Ps, dYs)], dim=1)
    return dX, dA, dB


def _clip(g, max_norm):
    norm = g.double().square().sum().sqrt()  # 64 bits: a sum over tens of millions of squares
    return norm.float().reshape(1), torch.clamp(max_norm / norm, max=1.0).float().reshape(1)


def _adamw(p, g, m, v, coef):
    g = g * coef
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    p = p * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    return p, m, v, p.to(torch.bfloat16)


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "serve":
        return [torch.cat([Y for Y, _ in _forwards(s, i)], dim=1) for i in range(len(s["X"]))]
    if kind == "norm":
        return _clip(s["g"], s["max_norm"])
    if kind == "step":
        norm, coef = _clip(s["g"], s["max_norm"])
        return (norm, coef, *_adamw(s["p"], s["g"], s["m"], s["v"], coef))
    n, r = case["n"], case["r"]
    if kind == "grad":
        return _backward(s, [torch.where(_chosen(s["ids"], n, r), P.repeat(1, n), 0.0) for P in s["P"].split(r, 1)])
    Ys, Ps = zip(*_forwards(s, 0))
    Y = torch.cat(Ys, dim=1)
    if kind == "project":
        return Y, torch.cat([P.reshape(-1, n, r).sum(1) for P in Ps], dim=1)
    dX, dA, dB = _backward(s, Ps)
    g = torch.cat([dA.flatten(), dB.flatten()])
    norm, coef = _clip(g, s["max_norm"])
    return (Y, dX, norm, coef, *_adamw(s["p"], g, s["m"], s["v"], coef))


# ---------------------------------------------------------------- the framework's calls

def _copies(s):
    """The step updates in place: it runs on copies, so that a pass leaves its inputs as they were."""
    s["p_new"].copy_(s["p"]), s["m_new"].copy_(s["m"]), s["v_new"].copy_(s["v"])


def _own(s):
    import paper_2609_33977_amd as gm
    case, kind = s["case"], s["case"]["kind"]
    if kind == "serve":
        gm.gm_lora_plan(s["ids"], case["n"], s["plan"])
        for X, A, B, base, Y, widths in zip(s["X"], s["A"], s["B"], s["base"], s["Y"], s["widths"]):
            gm.gm_lora_fwd(X, A, B, s["scale"], s["plan"], base, Y, ws=s["ws"], widths=widths)
        return s["Y"]
    if kind in ("project", "grad", "tune"):
        X, A, B = s["X"][0], s["A"][0], s["B"][0]
        gm.gm_lora_plan(s["ids"], case["n"], s["plan"])
        if kind != "grad":
            gm.gm_lora_fwd(X, A, B, s["scale"], s["plan"], s["base"][0], s["Y"][0], s["P"], s["ws"],
                           widths=s["widths"][0])
        if kind == "project":
            return s["Y"][0], s["P"]
        gm.gm_lora_bwd(s["dY"], X, A, B, s["scale"], s["plan"], s["P"], s["dX_base"], s["dX"], s["dA"], s["dB"], s["ws"],
                       widths=s["widths"][0])
        if kind == "grad":
            return s["dX"], s["dA"], s["dB"]
    gm.gm_grad_norm(s["list"], s["max_norm"], s["norm"], s["coef"], s["norm_ws"])
    if kind == "norm":
        return s["norm"], s["coef"]
    _copies(s)
    gm.gm_adamw_list(s["list"], LR, BETA1, BETA2, EPS, DECAY, STEP, s["coef"])
    stepped = (s["norm"], s["coef"], s["p_new"], s["m_new"], s["v_new"], s["p16"])
    return stepped if kind == "step" else (s["Y"][0], s["dX"], *stepped)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- 64 bits

def _exact_linear(s, i, backward=False):
    """By adapter and part of the stack, over the tokens that chose the adapter."""
    X, A, B, ids, r = s["X"][i], s["A"][i], s["B"][i], s["ids"], s["case"]["r"]
    Y, low = s["base"][i].double(), torch.zeros(X.shape[0], A.shape[1], dtype=torch.float64, device=X.device)
    dX = s["dX_base"].double() if backward else None
    dA, dB = (torch.zeros(w.shape, dtype=torch.float64, device=X.device) for w in (A, B))
    for a in range(A.shape[0]):
        t = (ids == a).nonzero()
        c, first = float(s["scale"][a]), 0
        for k, width in enumerate(s["widths"][i]):
            ranks, outs = torch.arange(k * r, k * r + r, device=X.device), slice(first, first + width)
            first += width
            x, wa, wb = X[t[:, 0]].double(), A[a, ranks].double(), B[a, outs].double()
            low[t, ranks] = x @ wa.t()
            Y[t[:, 0], outs] += c * (low[t, ranks] @ wb.t())
            if backward:
                dy = s["dY"][t[:, 0], outs].double()
                kept = s["P"][t, ranks].double() if s["case"]["kind"] == "grad" else low[t, ranks]
                q = c * (dy @ wb)
                dX[t[:, 0]] += q @ wa
                dA[a, ranks] = q.t() @ x
                dB[a, outs] = c * (dy.t() @ kept)
    return Y, low, dX, dA, dB


def _exact_step(p, g, m, v, max_norm):
    p, g, m, v = p.double(), g.double(), m.double(), v.double()
    norm = torch.linalg.vector_norm(g)
    coef = 1.0 if float(norm) <= max_norm else max_norm / float(norm)
    g = coef * g
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g ** 2 * (1 - BETA2)
    rate = torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS
    p = p - LR * DECAY * p - LR * m / (1 - BETA1 ** STEP) / rate
    return norm.reshape(1), torch.tensor([coef], dtype=torch.float64), p, m, v, p


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "step"):
        if kind == "step":
            return _exact_step(s["p"], s["g"], s["m"], s["v"], s["max_norm"])
        zero = torch.zeros_like(s["g"], dtype=torch.float64)
        return _exact_step(zero, s["g"], zero, zero, s["max_norm"])[:2]
    if kind == "serve":
        return [_exact_linear(s, i)[0] for i in range(len(s["X"]))]
    Y, low, dX, dA, dB = _exact_linear(s, 0, kind != "project")
    if kind == "project":
        return Y, low
    if kind == "grad":
        return dX, dA, dB
    return (Y, dX, *_exact_step(s["p"], torch.cat([dA.flatten(), dB.flatten()]), s["m"], s["v"], s["max_norm"]))


# ---------------------------------------------------------------- floors

def work(case):
    kind = case["kind"]
    if kind in ("norm", "step"):
        values = case["tensors"] * case["most"] * 9 / 16  # sizes are spread evenly from an eighth of the largest up
        if kind == "norm":
            return {"bytes": values * (2 if case["bf16"] else 4), "flops": 2 * values}
        return {"bytes": values * (16 + 12 + 2), "flops": 16 * values}
    T, n, r = case["T"], case["n"], case["r"]
    with_adapter = T * (1 - case["none"])
    used = n if case["runs"] else n * (1 - (1 - (1 - case["none"]) / n) ** T)  # adapters that some token chose
    nbytes = flops = 0
    for d_in, outs in _groups(case):
        weights = sum(2 * used * r * (d_in + o) for o in outs)
        if kind != "grad":
            nbytes += weights + 2 * T * d_in + 4 * T * sum(outs)  # weights, X, base read; Y written
            flops += sum(2 * with_adapter * r * (d_in + o) for o in outs)
        if kind == "project":
            nbytes += 4 * T * r * len(outs)
        if kind in ("grad", "tune"):
            # X, dY, base, P and weights read; dX, dA, dB written
            nbytes += weights + 2 * T * (3 * d_in + sum(outs)) + 4 * T * r * len(outs) + 2 * weights
            flops += sum(4 * with_adapter * r * (d_in + o) for o in outs)
        if kind == "tune":
            values = n * r * (len(outs) * d_in + sum(outs))
            nbytes += 30 * values
            flops += 16 * values
    return {"bytes": nbytes, "flops": flops}
