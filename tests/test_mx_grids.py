"""The 4-bit operators' launches at the ends of their ranges: a launch holds fewer than 2^32 work-items.  And the most matrices of a call."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._mx_launches import experts, products, program

compiled = pytest.mark.skipif(program() is None, reason="hipcc not available")
MOST = 1 << 18


@compiled
def test_products():
    shapes = [(M, N, K, act, y) for M in (1, 64, 300, 65536, MOST) for N in (1, 300, 65536, MOST) for K in (1, 128, 300, 4096, MOST) for act in (0, 2) for y in (0, 1)]
    for s, p in zip(shapes, products(*shapes)):
        assert 1 <= p.groups and p.groups * p.block < 1 << 32, (s, p)


@compiled
def test_experts():
    shapes = [(T, H, F, E, k, act, w, T) for T, k in ((1, 1), (1, 16), (512, 16), (8192, 1)) for H in (64, 32768) for F in (64, 32768) for E in (16, 512)
              for act in (0, 2) for w in (B.DTYPE_BF16, B.DTYPE_MXFP4)]
    for s, found in zip(shapes, experts(*shapes)):
        for p in found:
            assert 1 <= p.groups <= 3 * 256 and 1 <= p.most <= 16 and p.steps >= p.most, (s, p)


@pytest.mark.gpu
@pytest.mark.parametrize("down", [False, True])
def test_most_matrices(lib, down):
    n = 65535
    X = torch.randn((n, 3, 5), device="cuda")
    mx, values = B.MxMatrix(5 if down else 3, 3 if down else 5, n), torch.empty((n, 3, 5), dtype=torch.bfloat16, device="cuda")
    B.mx_quantize(X, mx, values=values, down=down)
    pick = [0, 1, 32768, n - 1]
    some, want = B.MxMatrix(mx.rows, mx.K, len(pick)), torch.empty((len(pick), 3, 5), dtype=torch.bfloat16, device="cuda")
    B.mx_quantize(X[pick], some, values=want, down=down)
    assert torch.equal(mx.codes[pick], some.codes) and torch.equal(mx.scales[pick], some.scales) and torch.equal(values[pick], want)
    with pytest.raises(B.Mlp2Error):
        B.mx_quantize(X[:1].repeat(n + 1, 1, 1), B.MxMatrix(mx.rows, mx.K, n + 1), down=down)
