"""MXFP4 quantisation on the GPU against the fp64 oracle: codes, scales and values are equal, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as M
from paper_2607_07862_amd import binding as B
from tests._train import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(X, down=False):
    """X [count, rows, cols] on the GPU, rows of any stride."""
    count, rows, cols = X.shape
    n, K = (cols, rows) if down else (rows, cols)
    mx = B.MxMatrix(n, K, count)
    mx.codes.fill_(0xA5), mx.scales.fill_(0x5A)
    values = torch.full((count, rows, cols), 7.0, dtype=BF, device="cuda")
    B.mx_quantize(X, mx, values=values, down=down)
    x = f64(X)
    for m in range(count):
        codes, scales, want = M.quantise(x[m].T if down else x[m])
        packed, s = M.pack(codes, scales)
        assert (mx.scales[m].cpu().numpy() == s).all(), "scales"
        bad = mx.codes[m].cpu().numpy() != packed
        assert not bad.any(), f"{int(bad.sum())} codes, first at {tuple(np.argwhere(bad)[0])}"
        want = want[:, :K].T if down else want[:, :K]
        got = f64(values[m])
        same = (got == want) & (np.signbit(got) == np.signbit(want)) | (np.isnan(got) & np.isnan(want))
        assert same.all(), f"value at {tuple(np.argwhere(~same)[0])}"
    # the same without values
    again = B.MxMatrix(n, K, count)
    B.mx_quantize(X, again, down=down)
    assert torch.equal(again.codes, mx.codes) and torch.equal(again.scales, mx.scales)


def numbers(gen, shape, dtype):
    """Values whose blocks differ in size, with exact ties, powers of two and zeros among them."""
    x = torch.randn(shape, generator=gen) * torch.exp(2 * torch.randn(shape[:-1] + (1,), generator=gen))
    pick = torch.rand(shape, generator=gen)
    x = torch.where(pick < 0.3, torch.randint(-28, 29, shape, generator=gen) * 0.25, x)
    x = torch.where(pick > 0.95, torch.zeros(()), x)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("down", [False, True])
@pytest.mark.parametrize("count,rows,cols", [(1, 1, 1), (1, 1, 32), (2, 3, 31), (1, 33, 128), (1, 5, 129), (3, 7, 33), (1, 70, 260), (1, 300, 64),
                                             (2, 129, 97), (1, 1, 1000), (1, 1025, 3), (1, 64, 513)])
def test_sizes(lib, count, rows, cols, down, dtype):
    gen = torch.Generator().manual_seed(rows * cols)
    check(numbers(gen, (count, rows, cols), dtype).cuda(), down)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("down", [False, True])
@pytest.mark.parametrize("pad,offset", [(1, 0), (7, 3), (64, 1)])
def test_rows_of_any_stride_and_start(lib, pad, offset, down, dtype):
    gen = torch.Generator().manual_seed(pad)
    wide = numbers(gen, (2, 37, 131 + pad + offset), dtype).cuda()
    check(wide[:, :, offset:offset + 131], down)
    check(wide[:, 3:30, offset:offset + 64], down)  # matrices further apart than their rows are long


@pytest.mark.parametrize("down", [False, True])
def test_extremes(lib, down):
    """The ends of the exponents' range, subnormal numbers, NaN, infinities and zeros of either sign."""
    gen = torch.Generator().manual_seed(5)
    for dtype, powers in ((F32, (-149, -140, -130, -128, -127, -126, -125, -124, -1, 0, 126, 127)), (BF, (-133, -130, -127, -126, -125, 0, 127))):
        x = torch.zeros((1, 32 * len(powers), 32), dtype=torch.float64)
        for i, p in enumerate(powers):
            x[0, 32 * i:32 * i + 32] = torch.ldexp(torch.rand((32, 32), generator=gen, dtype=torch.float64) * 4 - 2, torch.tensor(p)).clamp(-3.38e38, 3.38e38)
        x[0, 3, 4], x[0, 70, 1], x[0, 71, 2], x[0, 40, 5] = float("nan"), float("inf"), float("-inf"), -0.0
        check(x.to(dtype).cuda(), down)
        check(torch.zeros((1, 40, 50), dtype=dtype).neg().cuda(), down)


def test_large_offsets(lib):
    """Rows whose bytes lie beyond 4 GB from the first."""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("not enough memory")
    base = torch.empty(3 * (1 << 30), dtype=BF, device="cuda")
    X = base.as_strided((1, 3, 96), (3 << 30, (1 << 30) + 1, 1))
    X.copy_(numbers(torch.Generator().manual_seed(1), (1, 3, 96), BF))
    check(X[:, :, :96])
    check(X[:, :, :96], down=True)


def test_two_dimensions_nothing_and_streams(lib):
    X = torch.randn((40, 200), device="cuda")
    a, b = B.MxMatrix(40, 200), B.MxMatrix(40, 200, 1)
    B.mx_quantize(X, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.mx_quantize(X.unsqueeze(0), b, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    B.mx_quantize(X[:0], B.MxMatrix(0, 200))
    B.mx_quantize(X[:, :0], B.MxMatrix(40, 0))
    B.mx_quantize(X[:0], B.MxMatrix(200, 0), down=True)


def test_captured(lib):
    """A captured quantisation replays on new inputs."""
    X = torch.randn((65, 300), device="cuda").to(BF)
    mx, want = B.MxMatrix(65, 300), B.MxMatrix(65, 300)
    B.mx_quantize(X, mx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mx_quantize(X, mx)
    for i in range(4):
        X.normal_()
        mx.codes.zero_(), mx.scales.zero_()
        graph.replay()
        B.mx_quantize(X, want)
        torch.cuda.synchronize()
        assert torch.equal(mx.codes, want.codes) and torch.equal(mx.scales, want.scales), i
