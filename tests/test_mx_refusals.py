"""What the MXFP4 entry points refuse: on the CPU what is checked before any device call, on the GPU the calls of real plans."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from test_train_refusals import clib, refused  # noqa: F401

P = 1 << 20  # an aligned address that nothing reads


@pytest.mark.parametrize("args,code", [
    ((0, 64, 64, 0, 0), B.ERR_INVALID_ARG),
    ((8, 0, 64, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, -1, 0, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 3, 0), B.ERR_INVALID_ARG),
    ((8, 64, 64, 0, 2), B.ERR_INVALID_ARG),
    (((1 << 18) + 1, 64, 64, 0, 0), B.ERR_UNSUPPORTED),
    ((8, (1 << 18) + 1, 64, 0, 0), B.ERR_UNSUPPORTED),
    ((8, 64, (1 << 18) + 1, 0, 1), B.ERR_UNSUPPORTED),
])
def test_plans_refuse_before_touching_a_device(clib, args, code):  # noqa: F811
    assert not clib.mlp2_mx_plan(*args)
    assert clib.mlp2_last_error() == code


@pytest.mark.parametrize("change,code", [
    ({0: -1}, B.ERR_INVALID_ARG), ({1: -1}, B.ERR_INVALID_ARG), ({2: -1}, B.ERR_INVALID_ARG), ({3: 2}, B.ERR_INVALID_ARG), ({5: 2}, B.ERR_INVALID_ARG),
    ({0: 65536}, B.ERR_UNSUPPORTED), ({1: (1 << 20) + 1}, B.ERR_UNSUPPORTED),
    ({6: (1 << 40) + 1}, B.ERR_UNSUPPORTED), ({7: (1 << 40) + 1}, B.ERR_UNSUPPORTED),
    ({4: None}, B.ERR_INVALID_ARG), ({8: None}, B.ERR_INVALID_ARG), ({9: None}, B.ERR_INVALID_ARG),
    ({6: 63}, B.ERR_INVALID_ARG), ({7: 64 * 3}, B.ERR_INVALID_ARG),
    ({4: P + 1}, B.ERR_ALIGNMENT), ({8: 9 * P + 8}, B.ERR_ALIGNMENT), ({9: 17 * P + 4}, B.ERR_ALIGNMENT), ({10: 25 * P + 1}, B.ERR_ALIGNMENT),
    ({8: P}, B.ERR_INVALID_ARG), ({9: 9 * P + 16}, B.ERR_INVALID_ARG), ({10: 9 * P}, B.ERR_INVALID_ARG), ({10: P}, B.ERR_INVALID_ARG),
    ({0: 1000, 1: 1 << 20, 2: 128, 6: 128, 7: 128 << 20, 8: 1 << 45, 9: 1 << 46, 10: 1 << 47}, None),
])
def test_quantize_refuses(clib, change, code):  # noqa: F811
    """count, rows, cols, down, X, dtype, ldx, matrix_stride, codes, scales, values, stream."""
    args = [2, 4, 64, 0, P, 0, 64, 256, 9 * P, 17 * P, 25 * P, None]
    for i, v in change.items():
        args[i] = v
    if code is None:  # more pieces than a launch holds: found after the device is known
        assert clib.mlp2_mx_quantize(*args) in (B.ERR_DEVICE, B.ERR_HIP, B.ERR_UNSUPPORTED)
    else:
        assert clib.mlp2_mx_quantize(*args) == code


def test_nothing_to_quantise(clib):  # noqa: F811
    for i in range(3):
        args = [2, 4, 64, 0, None, 0, 64, 256, None, None, None, None]
        args[i] = 0
        assert clib.mlp2_mx_quantize(*args) == B.OK


def test_null_plan(clib):  # noqa: F811
    assert clib.mlp2_mx_product(None, 1, P, P, P, P, P, None) == B.ERR_INVALID_ARG
    clib.mlp2_mx_destroy(None)


@pytest.mark.gpu
def test_product_calls(lib):
    M, N, K = 8, 40, 200
    plan = B.MxPlan(M, N, K, B.ACT_SWIGLU)
    A, W, Y = B.MxMatrix(M, K), B.MxMatrix(N, K, 2), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    for m in (A, W):
        m.codes.zero_(), m.scales.zero_()
    plan.product(A, W, Y)
    with pytest.raises(TypeError):
        plan.product(A.codes, W, Y)
    with pytest.raises(TypeError):
        plan.product(A, W, Y.float())
    for a, w, y in ((B.MxMatrix(M, K + 1), W, Y), (A, B.MxMatrix(N, K), Y), (A, B.MxMatrix(N + 1, K, 2), Y), (A, W, Y[:-1]), (A, W, Y.t()), (A, W, Y.cpu())):
        with pytest.raises(ValueError):
            plan.product(a, w, y)
    big = B.MxMatrix(M + 1, K)
    refused(B.ERR_INVALID_ARG, plan.product, big, W, torch.empty((M + 1, N), dtype=torch.bfloat16, device="cuda"))
    refused(B.ERR_INVALID_ARG, plan.product, A, W, A.codes.view(-1)[:2 * M * N].view(torch.bfloat16).view(M, N))
    p = [t.data_ptr() for t in (A.codes, A.scales, W.codes, W.scales, Y)]
    for i in range(5):
        for v, code in ((None, B.ERR_INVALID_ARG), (p[i] + 1, B.ERR_ALIGNMENT)):
            args = list(p)
            args[i] = v
            assert B.load().mlp2_mx_product(plan.handle, M, *args, None) == code
    with pytest.raises(TypeError):
        B.MxPlan(M, N, K, 0, torch.float16)


@pytest.mark.gpu
def test_matrices_and_quantize_calls(lib):
    X = torch.zeros((6, 130), device="cuda")
    mx = B.MxMatrix(6, 130)
    B.mx_quantize(X, mx)
    with pytest.raises(TypeError):
        B.mx_quantize(X.half(), mx)
    for bad in (X[0], X[None, None], X.cpu(), X[:5], X[:, :129], X.t().contiguous().t(), X[:1].expand(6, 130), X.view(130, 6)):
        with pytest.raises(ValueError):
            B.mx_quantize(bad, mx)
    with pytest.raises(ValueError):
        B.mx_quantize(X, mx, down=True)
    with pytest.raises(TypeError):
        B.mx_quantize(X, mx, values=X)
    with pytest.raises(ValueError):
        B.mx_quantize(X, mx, values=torch.empty((6, 129), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        B.mx_quantize(X, mx.codes)
    with pytest.raises(TypeError):
        B.MxMatrix.of(mx.codes.int(), mx.scales, 130)
    for codes, scales, K in ((mx.codes[0], mx.scales, 130), (mx.codes, mx.scales, 128), (mx.codes, mx.scales[:, :1], 130), (mx.codes.cpu(), mx.scales.cpu(), 130),
                             (mx.codes[:, :, ::2], mx.scales, 130)):
        with pytest.raises(ValueError):
            B.MxMatrix.of(codes, scales, K)
    same = B.MxMatrix.of(mx.codes, mx.scales, 130)
    assert same.rows == 6 and same.count == 1 and same.codes.data_ptr() == mx.codes.data_ptr()
