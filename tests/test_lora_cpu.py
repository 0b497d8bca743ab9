"""Low-rank adapters and tensor lists without a GPU: the oracle's gradients against differences of its forward, sizes
of plans and workspaces, and every refusal of the entry points (nothing is launched, no pointer followed)."""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2609_33977_amd as gm

FAKE = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 4)
BIG = 1 << 40


def _case(seed=3, T=9, n=3, d_in=10, widths=(4, 7), r=3):
    g = np.random.default_rng(seed)
    ids = g.integers(-1, n, T)
    R, d_out = r * len(widths), sum(widths)
    return (g.normal(size=(T, d_in)), g.normal(size=(n, R, d_in)), g.normal(size=(n, d_out, r)), g.uniform(0.5, 2, n), ids,
            g.normal(size=(T, d_out)), widths, g.normal(size=(T, d_out)))


def test_oracle_forward_token_by_token():
    X, A, B, scale, ids, base, widths, _ = _case()
    Y, P = oracle.lora_fwd(X, A, B, scale, ids, base, widths)
    r, edges = B.shape[2], np.concatenate([[0], np.cumsum(widths)])
    for t, a in enumerate(ids):
        want = base[t].copy()
        if a >= 0:
            for k in range(len(widths)):
                low = A[a, k * r:(k + 1) * r] @ X[t]
                assert np.allclose(P[t, k * r:(k + 1) * r], low, rtol=1e-13, atol=1e-13)
                want[edges[k]:edges[k + 1]] += scale[a] * B[a, edges[k]:edges[k + 1]] @ low
        else:
            assert not P[t].any()
        assert np.allclose(Y[t], want, rtol=1e-13, atol=1e-13)


def test_oracle_gradients_against_differences():
    # the loss sum(dY Y) is linear in each of X, A and B alone: central differences are exact up to rounding
    X, A, B, scale, ids, base, widths, dY = _case()
    _, P = oracle.lora_fwd(X, A, B, scale, ids, base, widths)
    dX, dA, dB, _ = oracle.lora_bwd(dY, X, A, B, scale, ids, np.zeros_like(X), P, widths)
    loss = lambda x, a, b: float(np.sum(dY * oracle.lora_fwd(x, a, b, scale, ids, base, widths)[0]))  # noqa: E731
    for k, (w, grad) in enumerate(((X, dX), (A, dA), (B, dB))):
        for i in np.random.default_rng(k).choice(w.size, 40, replace=False):
            step = np.zeros(w.size)
            step[i] = 0.5
            lo, hi = ([v if j != k else v + s * step.reshape(w.shape) for j, v in enumerate((X, A, B))] for s in (-1, 1))
            assert abs(loss(*hi) - loss(*lo) - grad.flat[i]) < 1e-10


def test_oracle_norm():
    assert oracle.grad_norm([np.array([3.0]), np.array([[4.0]])], 10.0) == (5.0, 1.0)
    assert oracle.grad_norm([np.array([3.0, 4.0])], 1.0) == (5.0, 0.2)
    assert oracle.grad_norm([np.array([np.inf])], 1.0)[1] == 0.0
    assert oracle.grad_norm([np.array([np.nan])], 1.0)[1] == 0.0


def _widths(*w):
    return (ctypes.c_int64 * len(w))(*w)


@pytest.mark.parametrize("T,n", [(0, 1), (-1, 1), (262145, 1), (1, 0), (1, 2049), (1, -3)])
def test_plan_refuses_sizes(T, n):
    out = ctypes.c_size_t(0)
    assert gm.LIB.gm_lora_plan_size(T, n, ctypes.byref(out)) == gm.GM_ERR_SHAPE
    assert gm.LIB.gm_lora_plan(FAKE, T, n, FAKE, BIG, None) == gm.GM_ERR_SHAPE


def test_plan_refusals():
    L = gm.LIB
    need = gm.gm_lora_plan_size(100, 5)
    assert L.gm_lora_plan_size(100, 5, None) == gm.GM_ERR_NULL
    assert L.gm_lora_plan(None, 100, 5, FAKE, BIG, None) == gm.GM_ERR_NULL
    assert L.gm_lora_plan(FAKE, 100, 5, None, BIG, None) == gm.GM_ERR_NULL
    assert L.gm_lora_plan(FAKE, 100, 5, ODD, BIG, None) == gm.GM_ERR_ALIGN
    assert L.gm_lora_plan(ctypes.c_void_p((1 << 20) + 2), 100, 5, FAKE, BIG, None) == gm.GM_ERR_ALIGN
    assert L.gm_lora_plan(FAKE, 100, 5, FAKE, need - 1, None) == gm.GM_ERR_WORKSPACE


SHAPES = [  # d_in, widths, r
    (0, (64,), 16), (12, (64,), 16), (1 << 19, (64,), 16), (64, (), 16), (64, (64,) * 5, 16), (64, (64, 0), 16),
    (64, (64, 12), 16), (64, (1 << 18, 8), 16), (64, (64,), 0), (64, (64,), 4), (64, (64,), 20), (64, (64,), 136),
    (64, (-8,), 16),
]


def _fwd(X=FAKE, ldx=64, A=FAKE, B=FAKE, scale=FAKE, plan=FAKE, plan_bytes=BIG, T=10, n=2, d_in=64, widths=(64,), r=16,
         base=FAKE, ldb=None, Y=FAKE, ldy=None, P=FAKE, ws=FAKE, ws_bytes=BIG):
    w = _widths(*widths) if widths is not None else None
    ld = max(8, sum(widths or (8,)))
    return gm.LIB.gm_lora_fwd(X, ldx, A, B, scale, plan, plan_bytes, T, n, d_in, w, len(widths or (1,)), r, base,
                              ld if ldb is None else ldb, Y, ld if ldy is None else ldy, P, ws, ws_bytes, None)


def _bwd(dY=FAKE, lddy=None, X=FAKE, ldx=64, A=FAKE, B=FAKE, scale=FAKE, plan=FAKE, plan_bytes=BIG, P=FAKE, T=10, n=2,
         d_in=64, widths=(64,), r=16, base=FAKE, ldb=64, dX=FAKE, lddx=64, dA=FAKE, dB=FAKE, ws=FAKE, ws_bytes=BIG):
    w = _widths(*widths) if widths is not None else None
    ld = max(8, sum(widths or (8,)))
    return gm.LIB.gm_lora_bwd(dY, ld if lddy is None else lddy, X, ldx, A, B, scale, plan, plan_bytes, P, T, n, d_in, w,
                              len(widths or (1,)), r, base, ldb, dX, lddx, dA, dB, ws, ws_bytes, None)


@pytest.mark.parametrize("d_in,widths,r", SHAPES)
def test_linears_refuse_shapes(d_in, widths, r):
    out = ctypes.c_size_t(0)
    for op in (gm.GM_OP_FWD, gm.GM_OP_BWD):
        assert gm.LIB.gm_lora_workspace_size(op, 10, 2, d_in, _widths(*widths), len(widths), r,
                                             ctypes.byref(out)) == gm.GM_ERR_SHAPE
    ld = max(d_in, 64)
    assert _fwd(d_in=d_in, widths=widths, r=r, ldx=ld) == gm.GM_ERR_SHAPE
    assert _bwd(d_in=d_in, widths=widths, r=r, ldx=ld, ldb=ld, lddx=ld) == gm.GM_ERR_SHAPE


def test_forward_refusals():
    for name in ("X", "A", "B", "scale", "plan", "base", "Y"):
        assert _fwd(**{name: None}) == gm.GM_ERR_NULL, name
    assert _fwd(widths=None) == gm.GM_ERR_NULL
    for name in ("X", "A", "B", "plan", "base", "Y", "P", "ws"):
        assert _fwd(**{name: ODD}) == gm.GM_ERR_ALIGN, name
    assert _fwd(scale=ctypes.c_void_p((1 << 20) + 2)) == gm.GM_ERR_ALIGN
    for name in ("ldx", "ldb", "ldy"):
        for bad in (56, 68, 0, -64, 1 << 33):
            assert _fwd(**{name: bad}) == gm.GM_ERR_SHAPE, (name, bad)
    assert _fwd(ldb=128) == gm.GM_ERR_SHAPE                                     # base is Y with another stride
    assert _fwd(T=0) == gm.GM_ERR_SHAPE and _fwd(n=0) == gm.GM_ERR_SHAPE
    assert _fwd(plan_bytes=gm.gm_lora_plan_size(10, 2) - 1) == gm.GM_ERR_WORKSPACE
    assert _fwd(ws=None) == gm.GM_ERR_WORKSPACE
    assert _fwd(ws_bytes=gm.gm_lora_workspace_size(gm.GM_OP_FWD, 10, 2, 64, 64, 16) - 1) == gm.GM_ERR_WORKSPACE


def test_backward_refusals():
    for name in ("dY", "X", "A", "B", "scale", "plan"):
        assert _bwd(**{name: None}) == gm.GM_ERR_NULL, name
    assert _bwd(base=None) == gm.GM_ERR_NULL and _bwd(P=None) == gm.GM_ERR_NULL
    for name in ("dY", "X", "A", "B", "plan", "P", "base", "dX", "dA", "dB", "ws"):
        assert _bwd(**{name: ODD}) == gm.GM_ERR_ALIGN, name
    for name in ("lddy", "ldx", "ldb", "lddx"):
        for bad in (56, 68, 1 << 33):
            assert _bwd(**{name: bad}) == gm.GM_ERR_SHAPE, (name, bad)
    assert _bwd(ws=None) == gm.GM_ERR_WORKSPACE
    assert _bwd(ws_bytes=gm.gm_lora_workspace_size(gm.GM_OP_BWD, 10, 2, 64, 64, 16) - 1) == gm.GM_ERR_WORKSPACE
    assert _bwd(plan_bytes=64) == gm.GM_ERR_WORKSPACE
    assert _bwd(dX=None, dA=None, dB=None, P=None, base=None, ws=None) == gm.GM_OK   # nothing asked for


def test_launch_limit():
    # (T + 63 min(n + 1, T)) / 64 tiles times d_in + d_out up to 2^27
    assert gm.gm_lora_workspace_size(gm.GM_OP_FWD, 262144 - 126, 1, 1 << 14, 1 << 14, 8) > 0
    out = ctypes.c_size_t(0)
    assert gm.LIB.gm_lora_workspace_size(gm.GM_OP_FWD, 262144, 1, 1 << 14, _widths(1 << 14), 1, 8,
                                         ctypes.byref(out)) == gm.GM_ERR_SHAPE


def test_workspace_op_and_null():
    out = ctypes.c_size_t(0)
    assert gm.LIB.gm_lora_workspace_size(5, 10, 2, 64, _widths(64), 1, 16, ctypes.byref(out)) == gm.GM_ERR_VALUE
    assert gm.LIB.gm_lora_workspace_size(0, 10, 2, 64, _widths(64), 1, 16, None) == gm.GM_ERR_NULL
    assert gm.LIB.gm_lora_workspace_size(0, 10, 2, 64, None, 1, 16, ctypes.byref(out)) == gm.GM_ERR_NULL


def test_binding_refuses_before_the_library():
    import torch
    bf, u8 = torch.bfloat16, torch.uint8
    X, A, B = torch.zeros(4, 64, dtype=bf), torch.zeros(2, 16, 64, dtype=bf), torch.zeros(2, 32, 16, dtype=bf)
    scale, base, big = torch.ones(2), torch.zeros(4, 32, dtype=bf), torch.zeros(1 << 20, dtype=u8)
    ok = dict(X=X, A=A, B=B, scale=scale, plan=big, base=base, Y=base.clone(), ws=big)
    bad = [dict(X=X.float()), dict(X=X[:, :32]), dict(A=A[:, :8].contiguous()), dict(B=B[:1].contiguous()), dict(scale=torch.ones(3)),
           dict(base=base[:, :16]), dict(Y=base.float()), dict(Y=base.t()), dict(P=torch.zeros(4, 8)), dict(ws=None),
           dict(plan=None), dict(widths=(16, 8)), dict(widths=(16, 16)), dict(widths=()), dict(X=X[:1].expand(4, 64)),
           dict()]  # the last: all as it should be, but on the CPU
    for b in bad:
        with pytest.raises(ValueError):
            gm.gm_lora_fwd(**(ok | b))
    with pytest.raises(ValueError):
        gm.gm_lora_plan(torch.zeros(4, dtype=torch.int64), 2, big)
    with pytest.raises(ValueError):
        gm.gm_lora_bwd(base, X, A, B, scale, big, None, dX=X, ws=big)
    with pytest.raises(ValueError):
        gm.gm_tensor_list([torch.zeros(4, dtype=torch.float16)], big)
    with pytest.raises(ValueError):
        gm.gm_tensor_list([torch.zeros(4)], big, p=[torch.zeros(5)], m=[torch.zeros(4)], v=[torch.zeros(4)])
    with pytest.raises(ValueError):
        gm.gm_tensor_list([torch.zeros(4)], big, p=[torch.zeros(4), torch.zeros(4)], m=[torch.zeros(4)], v=[torch.zeros(4)])
    with pytest.raises(ValueError):
        gm.gm_grad_norm(big, 1.0, torch.zeros(2), torch.zeros(1), big)


def _list_args(sizes, **change):
    n = len(sizes)
    ptrs = lambda role: (ctypes.c_void_p * max(n, 1))(*[(role * 64 + i + 1) << 20 for i in range(n)])  # noqa: E731
    a = dict(p=ptrs(0), g=ptrs(1), m=ptrs(2), v=ptrs(3), p16=ptrs(4), b16=None, numel=(ctypes.c_int64 * max(n, 1))(*sizes), n=n,
             list=FAKE, bytes=BIG, stream=None)
    return tuple((a | change).values())


def test_list_refusals():
    f = gm.LIB.gm_tensor_list
    ptr = lambda *v: (ctypes.c_void_p * len(v))(*v)  # noqa: E731
    ok, odd = 1 << 20, (1 << 20) + 2
    assert f(*_list_args([5], g=None)) == gm.GM_ERR_NULL
    assert f(*_list_args([5], list=None)) == gm.GM_ERR_NULL
    assert f(*_list_args([5], numel=None)) == gm.GM_ERR_NULL
    for name in ("p", "m", "v"):
        assert f(*_list_args([5], **{name: None})) == gm.GM_ERR_NULL, name
    for name in ("p", "g", "m", "v", "p16"):
        assert f(*_list_args([5, 5], **{name: ptr(ok, None)})) == gm.GM_ERR_NULL, name
    for name in ("p", "g", "m", "v"):
        assert f(*_list_args([5, 5], **{name: ptr(ok, odd)})) == gm.GM_ERR_ALIGN, name
    assert f(*_list_args([5], p16=ptr(ok + 1))) == gm.GM_ERR_ALIGN
    assert f(*_list_args([5], g=ptr(ok + 1), b16=(ctypes.c_uint8 * 1)(1))) == gm.GM_ERR_ALIGN
    assert f(*_list_args([-1])) == gm.GM_ERR_SHAPE and f(*_list_args([1 << 41])) == gm.GM_ERR_SHAPE
    assert f(*_list_args([])) == gm.GM_ERR_SHAPE
    assert f(*_list_args([1 << 40] * 9)) == gm.GM_ERR_SHAPE                      # more chunks than an int counts
    assert f(*_list_args([5], list=ODD)) == gm.GM_ERR_ALIGN
    assert f(*_list_args([5], bytes=gm.gm_tensor_list_size([5]) - 1)) == gm.GM_ERR_WORKSPACE


def test_list_refuses_shared_memory():
    # fake addresses: GM_ERR_DEVICE (no GPU here, or nothing launched there) would mean that the list was accepted
    f = gm.LIB.gm_tensor_list
    ptr = lambda *v: (ctypes.c_void_p * len(v))(*v)  # noqa: E731
    a = 1 << 30
    for name in ("p", "m", "v"):
        for second in (a, a + 4 * 99):                                           # the same buffer, or its last value
            assert f(*_list_args([100, 100], **{name: ptr(a, second)})) == gm.GM_ERR_VALUE
    assert f(*_list_args([100, 100], p16=ptr(a, a + 2 * 99))) == gm.GM_ERR_VALUE
    assert f(*_list_args([100], p=ptr(a), g=ptr(a))) == gm.GM_ERR_VALUE          # a gradient that is its parameter
    assert f(*_list_args([100], m=ptr(a), v=ptr(a + 200))) == gm.GM_ERR_VALUE
    big = _list_args([10, 1000, 10], g=ptr(1 << 40, a, a + 40), p=ptr(1 << 41, 1 << 42, a + 3996))
    assert f(*big) == gm.GM_ERR_VALUE                                            # inside a long gradient that began before


def test_norm_and_step_refusals():
    L, W = gm.LIB, gm.GM_GRAD_NORM_WORKSPACE_BYTES
    for args in ((None, BIG, 1.0, FAKE, FAKE, FAKE, W), (FAKE, BIG, 1.0, None, FAKE, FAKE, W), (FAKE, BIG, 1.0, FAKE, None, FAKE, W)):
        assert L.gm_grad_norm(*args, None) == gm.GM_ERR_NULL
    for bad in (0.0, -1.0, float("nan")):
        assert L.gm_grad_norm(FAKE, BIG, bad, FAKE, FAKE, FAKE, W, None) == gm.GM_ERR_VALUE
    assert L.gm_grad_norm(ODD, BIG, 1.0, FAKE, FAKE, FAKE, W, None) == gm.GM_ERR_ALIGN
    assert L.gm_grad_norm(FAKE, BIG, 1.0, FAKE, FAKE, ODD, W, None) == gm.GM_ERR_ALIGN
    assert L.gm_grad_norm(FAKE, BIG, 1.0, FAKE, FAKE, None, W, None) == gm.GM_ERR_WORKSPACE
    assert L.gm_grad_norm(FAKE, BIG, 1.0, FAKE, FAKE, FAKE, W - 1, None) == gm.GM_ERR_WORKSPACE
    assert L.gm_grad_norm(FAKE, 16, 1.0, FAKE, FAKE, FAKE, W, None) == gm.GM_ERR_WORKSPACE
    ok = (1e-3, 0.9, 0.999, 1e-8, 0.05, 1, None, None)
    assert L.gm_adamw_list(None, BIG, *ok) == gm.GM_ERR_NULL
    assert L.gm_adamw_list(ODD, BIG, *ok) == gm.GM_ERR_ALIGN
    assert L.gm_adamw_list(FAKE, 16, *ok) == gm.GM_ERR_WORKSPACE
    for i, bad in ((0, -1.0), (1, 1.0), (2, -0.1), (3, 0.0), (4, float("nan")), (5, 0)):
        assert L.gm_adamw_list(FAKE, BIG, *(bad if j == i else v for j, v in enumerate(ok))) == gm.GM_ERR_VALUE
