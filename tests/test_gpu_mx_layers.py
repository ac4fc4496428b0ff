"""4-bit matrices in a user's hands: the input's gradient of a layer without activation, and arrays of another layout brought to the library's."""
import numpy as np
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._mx_gpu import assert_near, held, product_and_tol

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("y", [BF, F32])
@pytest.mark.parametrize("M,K,N", [(1, 64, 96), (33, 200, 321), (150, 640, 1000)])
def test_input_gradient(lib, M, K, N, y):
    """Y = X W of W [K, N] has dX = dY W^T: a product over N, of dY and of W as it lies, both quantised along their rows."""
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    dY, W = torch.randn((M, N), generator=gen, device="cuda", dtype=BF), torch.randn((K, N), generator=gen, device="cuda", dtype=BF) * N**-0.5
    g, w, back = B.MxMatrix(M, N), B.MxMatrix(K, N), torch.empty_like(W)
    B.mx_quantize(dY, g)
    B.mx_quantize(W, w, values=back)
    dX = torch.full((M, K), float("nan"), dtype=y, device="cuda")
    B.MxPlan(M, K, N, B.ACT_IDENTITY, y).product(g, w, dX)
    ref, tol = product_and_tol(held(g), [held(w)], "identity", y == F32)
    assert_near(dX, ref, tol, "dX")
    # the same by differences: the layer X -> sum dY' (X W'), which is linear, along one direction
    v = torch.randn((M, K), generator=gen, device="cuda", dtype=torch.float64)
    f = lambda x: (held(g) * (x @ back.double())).sum()  # noqa: E731
    x = torch.randn((M, K), generator=gen, device="cuda", dtype=torch.float64)
    difference = (f(x + v) - f(x - v)) / 2
    assert (difference - (dX.double() * v).sum()).abs() <= (tol * v.abs()).sum() + 1e-9 * f(x).abs().clamp(min=1)


@pytest.mark.parametrize("rows,K,count", [(5, 32, 1), (37, 96, 2), (64, 128, 1), (9, 416, 3)])
def test_scales_by_rows(lib, rows, K, count):
    """Scales [count, rows, K / 32] and codes [count, rows, K / 2], K a multiple of 32, as ``MxMatrix.of`` says how to bring them over."""
    mx = B.MxMatrix(rows, K, count)
    B.mx_quantize(torch.randn((count, rows, K), device="cuda"), mx)
    own = mx.scales.transpose(1, 2).reshape(count, rows, -1)[:, :, :K // 32].contiguous()
    codes = mx.codes[:, :, :K // 2].contiguous()
    groups = -(-K // 128)
    pad = torch.nn.functional.pad
    scales = pad(own, (0, 4 * groups - K // 32)).view(count, rows, groups, 4).transpose(1, 2).contiguous()
    other = B.MxMatrix.of(pad(codes, (0, 64 * groups - K // 2)), scales, K)
    assert torch.equal(other.codes, mx.codes) and torch.equal(other.scales, mx.scales)
    assert np.array_equal(held(other).cpu().numpy(), held(mx).cpu().numpy())
