"""What the training operators refuse: on the CPU what is checked before any device call, on the GPU the calls of real plans."""
import ctypes
import os

import pytest
import torch

from paper_2607_07862_amd import binding as B


@pytest.fixture(scope="module")
def clib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2607_07862_amd import build

        build.build()
    return B.load()


@pytest.mark.parametrize("name,args,code", [
    ("train", (0, 128, 128, 0, 0), B.ERR_INVALID_ARG),
    ("train", (8, 0, 128, 0, 0), B.ERR_INVALID_ARG),
    ("train", (8, 128, -64, 0, 0), B.ERR_INVALID_ARG),
    ("train", (8, 128, 128, 3, 0), B.ERR_INVALID_ARG),
    ("train", (8, 128, 128, -1, 0), B.ERR_INVALID_ARG),
    ("train", (8, 128, 128, 0, B.DTYPE_F32), B.ERR_INVALID_ARG),
    ("train", (8, 100, 128, 0, 0), B.ERR_UNSUPPORTED),
    ("train", (8, 128, 130, 0, 0), B.ERR_UNSUPPORTED),
    ("train", ((1 << 20) + 1, 128, 128, 0, 0), B.ERR_UNSUPPORTED),
    ("train", (8, 1 << 19, 128, 0, 0), B.ERR_UNSUPPORTED),
    ("norm", (0, 128, 0, 0), B.ERR_INVALID_ARG),
    ("norm", (8, 0, 0, 0), B.ERR_INVALID_ARG),
    ("norm", (8, 128, 2, 0), B.ERR_INVALID_ARG),
    ("norm", (8, 128, 0, -1), B.ERR_INVALID_ARG),
    ("norm", (8, 16385, 0, 0), B.ERR_UNSUPPORTED),
    ("norm", ((1 << 24) + 1, 128, 0, 0), B.ERR_UNSUPPORTED),
    ("norm", (8, 128, B.DTYPE_BF16, B.DTYPE_F32), B.ERR_UNSUPPORTED),
    ("ortho", (0, 128, 128, 0), B.ERR_INVALID_ARG),
    ("ortho", (1, 0, 128, 0), B.ERR_INVALID_ARG),
    ("ortho", (1, 128, -1, 0), B.ERR_INVALID_ARG),
    ("ortho", (1, 128, 128, 2), B.ERR_INVALID_ARG),
    ("ortho", (4097, 128, 128, 0), B.ERR_UNSUPPORTED),
    ("ortho", (1, 65537, 128, 0), B.ERR_UNSUPPORTED),
])
def test_plans_refuse_before_touching_a_device(clib, name, args, code):
    assert not getattr(clib, f"mlp2_{name}_plan")(*args)
    assert clib.mlp2_last_error() == code


def test_null_plans(clib):
    p = 16
    one = (ctypes.c_float * 3)(1, 0, 0)
    assert clib.mlp2_train_forward(None, 1, p, p, p, p, p, None) == B.ERR_INVALID_ARG
    assert clib.mlp2_train_backward(None, 1, p, p, p, p, p, p, p, p, None) == B.ERR_INVALID_ARG
    assert clib.mlp2_norm_forward(None, 1, p, 8, p, p, 1e-5, p, 8, p, p, None) == B.ERR_INVALID_ARG
    assert clib.mlp2_norm_backward(None, 1, p, 8, p, 8, p, p, p, p, 8, p, p, None) == B.ERR_INVALID_ARG
    assert clib.mlp2_ortho_run(None, p, p, 1, one, 0.0, None) == B.ERR_INVALID_ARG
    for name in ("train", "norm", "ortho"):
        getattr(clib, f"mlp2_{name}_destroy")(None)


# ------------------------------------------------------------------ real plans


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


def refused(code, call, *args, **kw):
    with pytest.raises(B.Mlp2Error) as e:
        call(*args, **kw)
    assert e.value.code == code


@pytest.mark.gpu
def test_train_calls(lib):
    M, H, F = 16, 64, 128
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    X, W1, W2, P, Y = bf(M, H), bf(2, H, F), bf(F, H), bf(2, M, F), bf(M, H)
    plan.forward(X, W1, W2, P, Y)
    with pytest.raises(TypeError):
        plan.forward(X.float(), W1, W2, P, Y)
    with pytest.raises(ValueError):
        plan.forward(X.cpu(), W1, W2, P, Y)
    with pytest.raises(ValueError):
        plan.forward(X, W1[0], W2, P, Y)  # a gated layer has two first weights
    with pytest.raises(ValueError):
        plan.forward(X, W1, W2.t(), P, Y)
    with pytest.raises(ValueError):
        plan.forward(X[:, ::2], W1, W2, P, Y)
    refused(B.ERR_INVALID_ARG, plan.forward, bf(M + 1, H), W1, W2, bf(2, M + 1, F), bf(M + 1, H))  # more rows than planned
    refused(B.ERR_INVALID_ARG, plan.forward, X, W1, W2, P, X)  # Y over X
    flat = bf(M * H + 8)
    refused(B.ERR_ALIGNMENT, plan.forward, flat[1:M * H + 1].view(M, H), W1, W2, P, Y)
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, W1, W2, P)  # no gradient asked for
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, W1, W2, P, dX=Y)  # dX over dY
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, W1, W2, P, dW1=bf(2, H, F), dW2=W2)
    big = bf(3 * F, H)
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, W1, W2, P, dX=big[:M], dW2=big[8:8 + F])  # outputs over each other
    raw = [t.data_ptr() for t in (X, W1, W2, P, Y)]
    for i in range(5):
        args = list(raw)
        args[i] = None
        assert B.load().mlp2_train_forward(plan.handle, M, *args, None) == B.ERR_INVALID_ARG
    assert B.load().mlp2_train_forward(plan.handle, -1, *raw, None) == B.ERR_INVALID_ARG


@pytest.mark.gpu
def test_norm_calls(lib):
    M, H = 6, 40
    plan = B.NormPlan(M, H, torch.bfloat16)
    X, Y, w, st = bf(M, H), bf(M, H), torch.ones(H, device="cuda"), torch.ones(M, device="cuda")
    plan.forward(X, w, w, Y)
    with pytest.raises(TypeError):
        plan.forward(X.float(), w, w, Y)
    with pytest.raises(TypeError):
        plan.forward(X, w.bfloat16(), w, Y)
    with pytest.raises(ValueError):
        plan.forward(X, w[:-1], w, Y)
    with pytest.raises(ValueError):
        plan.forward(bf(H, M).t(), w, w, Y)  # columns apart
    with pytest.raises(ValueError):
        plan.forward(X[:1].expand(M, H), w, w, Y)  # rows over each other
    with pytest.raises(TypeError):
        B.NormPlan(M, H, torch.float16)
    refused(B.ERR_INVALID_ARG, plan.forward, X, w, w, Y, eps=-1.0)
    refused(B.ERR_INVALID_ARG, plan.forward, X, w, w, Y, eps=float("nan"))
    refused(B.ERR_INVALID_ARG, plan.forward, X, w, w, X)
    refused(B.ERR_INVALID_ARG, plan.forward, bf(M + 1, H), w, w, bf(M + 1, H))
    refused(B.ERR_INVALID_ARG, plan.forward, X, w, w, Y, st, st)  # mean over rstd
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, w, st, st.clone(), Y)
    refused(B.ERR_INVALID_ARG, plan.backward, Y, X, w, st, st.clone(), bf(M, H), w, None)
    p = [t.data_ptr() for t in (X, Y, w)]
    fwd = B.load().mlp2_norm_forward
    assert fwd(plan.handle, M, p[0], H - 1, p[2], p[2], 1e-5, p[1], H, None, None, None) == B.ERR_INVALID_ARG
    assert fwd(plan.handle, M, p[0] + 1, H, p[2], p[2], 1e-5, p[1], H, None, None, None) == B.ERR_ALIGNMENT
    assert fwd(plan.handle, M, None, H, p[2], p[2], 1e-5, p[1], H, None, None, None) == B.ERR_INVALID_ARG


@pytest.mark.gpu
def test_ortho_calls(lib):
    plan = B.OrthoPlan(2, 24, 40)
    G, O = torch.ones((2, 24, 40), device="cuda"), bf(2, 24, 40)
    plan.run(G, O)
    with pytest.raises(TypeError):
        plan.run(G.bfloat16(), O)
    with pytest.raises(TypeError):
        plan.run(G, O.float())
    with pytest.raises(ValueError):
        plan.run(G[0], O[0])
    with pytest.raises(ValueError):
        plan.run(G, O, steps=3, coeffs=[(1.0, 0.0, 0.0)] * 2)
    refused(B.ERR_INVALID_ARG, plan.run, G, O, steps=0)
    refused(B.ERR_INVALID_ARG, plan.run, G, O, steps=65)
    refused(B.ERR_INVALID_ARG, plan.run, G, O, eps=-1e-9)
    for bad in (float("nan"), float("inf"), 65.0):
        refused(B.ERR_INVALID_ARG, plan.run, G, O, coeffs=(bad, 0.0, 0.0))
    refused(B.ERR_INVALID_ARG, plan.run, G, G.view(torch.bfloat16)[:, :, :40].contiguous().new_empty(0).set_(G.view(torch.bfloat16).untyped_storage(), 0, (2, 24, 40), (960, 40, 1)))
