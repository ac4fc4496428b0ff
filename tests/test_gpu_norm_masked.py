"""Layer norm's backward pass where nothing is read: columns past a row's end and rows past the last take no part in any sum."""
import pytest
import torch

from oracle import train_oracle as T
from paper_2607_07862_amd import binding as B
from tests._train import U16, U32, assert_within, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("x,y", [(BF, BF), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("M,H", [(1, 1), (3, 7), (65, 64), (5, 900), (3, 2111), (300, 1000), (2, 8195), (3, 16384)])
def test_rows_of_one_large_value(lib, M, H, x, y):
    """Every x is the row's mean, so xhat is 0, dX = rstd (g - mean(g)) and dweight is 0; mean times rstd passes fp32's range,
    as it does in the places that hold no x.  Tolerances as for other rows: a few roundings of fp32, and the result's own."""
    gen = torch.Generator().manual_seed(M + H)
    large, scale = 2.0**110, 1e6  # (rstd for eps = 1e-12)
    X = torch.full((M, H), large, dtype=x, device="cuda")
    dY, w = torch.randn((M, H), generator=gen).to(y).cuda(), (1 + 0.2 * torch.randn(H, generator=gen)).cuda()
    mean, rstd = torch.full((M,), large, device="cuda"), torch.full((M,), scale, device="cuda")
    dX, dw, db = torch.empty_like(X), torch.full((H,), float("nan"), device="cuda"), torch.full((H,), float("nan"), device="cuda")
    B.NormPlan(M, H, x, y).backward(dY, X, w, mean, rstd, dX, dw, db)
    rX, r_dw, r_db = T.norm_backward(f64(dY), f64(X), f64(w), f64(mean), f64(rstd))
    assert not r_dw.any()
    g = abs(f64(dY) * f64(w))
    own = U16 if x == BF else 4 * U32
    assert_within(dX, rX, own * abs(rX) + scale * (g + g.mean(1, keepdims=True)) * 32 * U32, "dX")
    assert not dw.any()
    assert_within(db, r_db, (M + 16) * U32 * abs(f64(dY)).sum(0) + 1e-30, "dbias")
