"""What the mixture-of-experts entry points refuse: on the CPU what is checked before any device call, on the GPU real plans' calls."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from test_train_refusals import clib, refused  # noqa: F401

P = 1 << 20


@pytest.mark.parametrize("args,code", [
    ((0, 64, 64, 4, 2, 0, 0), B.ERR_INVALID_ARG),
    ((8, 0, 64, 4, 2, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, -64, 4, 2, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 0, 0, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 4, 5, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 4, 2, 3, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 4, 2, 0, B.DTYPE_F32), B.ERR_INVALID_ARG),
    ((8, 96, 64, 4, 2, 0, 0), B.ERR_UNSUPPORTED),
    ((8, 64, 100, 4, 2, 0, 0), B.ERR_UNSUPPORTED),
    ((8, 64, 32832, 4, 2, 0, 2), B.ERR_UNSUPPORTED),
    ((8, 64, 64, 513, 2, 0, 0), B.ERR_UNSUPPORTED),
    ((8, 64, 64, 40, 17, 0, 0), B.ERR_UNSUPPORTED),
    ((2049, 64, 64, 8, 4, 0, 0), B.ERR_UNSUPPORTED),
    ((1 << 62, 64, 64, 8, 4, 0, 0), B.ERR_UNSUPPORTED),
])
def test_plans_refuse_before_touching_a_device(clib, args, code):  # noqa: F811
    assert not clib.mlp2_moe_plan(*args)
    assert clib.mlp2_last_error() == code


def test_null_plan(clib):  # noqa: F811
    assert clib.mlp2_moe_forward(None, 1, P, P, 0, P, None, P, None, P, P, P, None) == B.ERR_INVALID_ARG
    assert clib.mlp2_moe_experts(None, 1, P, P, P, P, None, P, None, P, None) == B.ERR_INVALID_ARG
    clib.mlp2_moe_destroy(None)


def tensors(T, H, F, E, k, nb):
    bf, i32 = torch.bfloat16, torch.int32
    z = lambda *s, t=bf: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    return z(T, H), z(H, E), z(E, nb, H, F), z(E, F, H), z(T, H), z(T, k, t=i32), z(T, k, t=torch.float32)


@pytest.mark.gpu
def test_calls(lib):
    T, H, F, E, k = 6, 64, 128, 5, 2
    plan = B.MoePlan(T, H, F, E, k, B.ACT_SWIGLU)
    good = list(tensors(T, H, F, E, k, 2))
    plan.forward(*good)
    for i, bad, error in ((0, good[0].float(), TypeError), (0, good[0].cpu(), ValueError), (0, good[0][:, ::2], ValueError), (1, good[1].half(), TypeError),
                          (1, good[1].t(), ValueError), (1, good[1][:, :4], ValueError), (2, good[2][:, :1], ValueError), (2, good[2][:, 0], ValueError),
                          (3, good[3][:4], ValueError), (3, good[3].transpose(1, 2), ValueError), (4, good[4][:5], ValueError), (5, good[5].long(), TypeError),
                          (5, good[5][:, :1], ValueError), (6, good[6].bfloat16(), TypeError)):
        args = list(good)
        args[i] = bad
        with pytest.raises(error):
            plan.forward(*args)
    with pytest.raises(TypeError):
        plan.forward(*good[:2], B.MxMatrix(F, H, 2 * E), B.MxMatrix(H, F, E), *good[4:])
    with pytest.raises(TypeError):
        B.MoePlan(T, H, F, E, k, 0, "int4")
    with pytest.raises(TypeError):
        B.MoePlan(T, H, F, E, k, 0, torch.float32)
    more = tensors(T + 1, H, F, E, k, 2)
    refused(B.ERR_INVALID_ARG, plan.forward, more[0], *good[1:4], *more[4:])
    refused(B.ERR_INVALID_ARG, plan.forward, *good[:4], good[0], *good[5:])  # Y over X
    refused(B.ERR_INVALID_ARG, plan.forward, *good[:5], good[6].view(torch.int32), good[6])  # ids over gates
    refused(B.ERR_INVALID_ARG, plan.experts, good[0], good[5], good[6], good[2], good[3], good[0])
    p = [t.data_ptr() for t in good]
    call = B.load().mlp2_moe_forward
    raw = [p[0], p[1], 0, p[2], None, p[3], None, p[4], p[5], p[6], None]
    assert call(plan.handle, T, *raw) == B.OK
    for i in (0, 1, 3, 5, 7, 8, 9):
        for v, code in ((None, B.ERR_INVALID_ARG), (raw[i] + 1, B.ERR_ALIGNMENT)):
            args = list(raw)
            args[i] = v
            assert call(plan.handle, T, *args) == code, i
    for i, v in ((2, 2), (4, p[2]), (6, p[3])):  # a router of another type, scales with bf16 weights
        args = list(raw)
        args[i] = v
        assert call(plan.handle, T, *args) == B.ERR_INVALID_ARG
    assert call(plan.handle, -1, *raw) == B.ERR_INVALID_ARG
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_calls_with_quantised_weights(lib):
    T, H, F, E, k = 3, 64, 128, 4, 2
    plan = B.MoePlan(T, H, F, E, k, B.ACT_GELU_TANH, "mxfp4")
    X, Wr, _, _, Y, ids, gates = tensors(T, H, F, E, k, 1)
    W1, W2 = B.MxMatrix(F, H, E), B.MxMatrix(H, F, E)
    for m in (W1, W2):
        m.codes.zero_(), m.scales.zero_()
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    for w1, w2 in ((B.MxMatrix(F, H, 2 * E), W2), (B.MxMatrix(H, F, E), W2), (W1, B.MxMatrix(H, F, E - 1)), (W1, B.MxMatrix(F, H, E))):
        with pytest.raises(ValueError):
            plan.forward(X, Wr, w1, w2, Y, ids, gates)
    with pytest.raises(TypeError):
        plan.experts(X, ids, gates, W1.codes, W2, Y)
    p = [X.data_ptr(), ids.data_ptr(), gates.data_ptr(), W1.codes.data_ptr(), None, W2.codes.data_ptr(), W2.scales.data_ptr(), Y.data_ptr(), None]
    assert B.load().mlp2_moe_experts(plan.handle, T, *p) == B.ERR_INVALID_ARG  # no scales
    torch.cuda.synchronize()
