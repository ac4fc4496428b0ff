"""Layer norm at the end of fp32's range: what the header says of rows whose sums leave it, and rows just inside."""
import pytest
import torch

from oracle import train_oracle as T
from paper_2607_07862_amd import binding as B
from tests._train import U32, f64

pytestmark = pytest.mark.gpu


def test_sums_past_fp32(lib):
    M, H = 4, 512
    gen = torch.Generator().manual_seed(0)
    X = torch.randn((M, H), generator=gen)
    X[1] *= 1e25   # the sum of squares overflows
    X[2] = 1e37    # the sum does
    X[3] *= 1e17   # neither
    X = X.cuda()
    w, b = torch.rand(H, generator=gen).cuda(), torch.rand(H, generator=gen).cuda()
    Y, mean, rstd = torch.empty_like(X), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    B.NormPlan(M, H, torch.float32).forward(X, w, b, Y, mean, rstd)
    assert rstd[1] == 0 and torch.equal(Y[1], b) and Y[2].isnan().all()
    for i in (0, 3):
        ref, _, r = T.norm_forward(f64(X[i:i + 1]), f64(w), f64(b), 1e-5)
        assert abs(f64(rstd[i:i + 1]) - r) <= 64 * U32 * r
        assert (abs(f64(Y[i:i + 1]) - ref) <= 64 * U32 * (abs(ref) + abs(f64(b)) + 8)).all()
