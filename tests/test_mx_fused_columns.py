"""Quantisation of matrices that are columns of one buffer: a fused weight ``[K, 2 N]`` seen as two ``[K, N]``."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from test_train_refusals import clib  # noqa: F401

P = 1 << 20
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("count,rows,cols,ldx,stride", [(2, 4, 64, 128, 64), (3, 4, 64, 200, 65), (5, 100, 7, 35, 7), (2, 4, 64, 200, 100)])
def test_accepted_up_to_the_device(clib, count, rows, cols, ldx, stride):  # noqa: F811
    """Refused for the lack of a GPU alone."""
    args = [count, rows, cols, 0, P, 0, ldx, stride, 1 << 40, 1 << 41, 1 << 42, None]
    if torch.cuda.is_available():
        pytest.skip("would be launched")
    assert clib.mlp2_mx_quantize(*args) in (B.ERR_DEVICE, B.ERR_HIP)


@pytest.mark.parametrize("count,rows,cols,ldx,stride", [(2, 4, 64, 127, 64), (3, 4, 64, 191, 64), (2, 4, 64, 128, 63), (2, 4, 64, 128, 65), (2, 4, 64, 128, 0), (2, 4, 64, 128, -64)])
def test_matrices_that_share_elements_are_refused(clib, count, rows, cols, ldx, stride):  # noqa: F811
    args = [count, rows, cols, 0, P, 0, ldx, stride, 1 << 40, 1 << 41, 1 << 42, None]
    assert clib.mlp2_mx_quantize(*args) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("codes,scales,values", [(P + 4 * 128 * 2 - 16, 1 << 41, 1 << 42), (1 << 40, P, 1 << 42), (1 << 40, 1 << 41, P + 126)])
def test_outputs_over_the_buffer_are_refused(clib, codes, scales, values):  # noqa: F811
    args = [2, 4, 64, 0, P, 0, 128, 64, codes, scales, values, None]
    assert clib.mlp2_mx_quantize(*args) == B.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("down", [False, True])
@pytest.mark.parametrize("count,rows,cols,pad", [(2, 70, 260, 0), (3, 33, 37, 0), (2, 129, 64, 5), (4, 1, 31, 2)])
def test_equals_the_copied_matrices(lib, count, rows, cols, pad, down, dtype):
    gen = torch.Generator().manual_seed(rows)
    wide = (torch.randn((rows, count * (cols + pad)), generator=gen) * 3).to(dtype).cuda()
    X = wide.view(rows, count, cols + pad).transpose(0, 1)[:, :, :cols]  # [count, rows, cols]: columns of `wide`
    before = wide.clone()
    out = []
    for x in (X, X.contiguous()):
        mx = B.MxMatrix(cols if down else rows, rows if down else cols, count)
        values = torch.full((count, rows, cols), 7.0, dtype=BF, device="cuda")
        B.mx_quantize(x, mx, values=values, down=down)
        out.append((mx.codes, mx.scales, values))
    assert all(torch.equal(a, b) for a, b in zip(*out)) and torch.equal(wide, before)


@pytest.mark.gpu
def test_shared_elements(lib):
    x = torch.zeros(1000, device="cuda")
    for strides in ((32, 65, 1), (64, 127, 1), (0, 128, 1)):
        with pytest.raises(ValueError):
            B.mx_quantize(x.as_strided((2, 4, 64), strides), B.MxMatrix(4, 64, 2))
