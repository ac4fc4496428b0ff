"""Training passes on tensors beyond 4 GB: offsets of 64 bits in every operand with a row or plane index."""
import pytest
import torch

from paper_2607_07862_amd import binding as B

pytestmark = pytest.mark.gpu


def test_mlp_tensors_beyond_4_gb(lib):
    """330000 rows of 64 through 2 x 8192: P is 10.8 GB (its second plane starts past 4 GB), dP rows reach 10.8 GB, Z 5.4 GB.
    Rows at both ends and at the 4 GB marks against 64 bits; the weight gradients against 64-bit sums over all rows."""
    M, H, F = 330001, 64, 8192
    gen = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    X, W1, W2, dY = normal(M, H), normal(2, H, F) * H**-0.5, normal(F, H) * F**-0.5, normal(M, H)
    P, Y = torch.empty((2, M, F), dtype=torch.bfloat16, device="cuda"), torch.empty_like(X)
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    plan.forward(X, W1, W2, P, Y)
    dX, dW1, dW2 = torch.empty_like(X), torch.empty_like(W1), torch.empty_like(W2)
    plan.backward(dY, X, W1, W2, P, dX, dW1, dW2)
    torch.cuda.synchronize()
    w1, w2 = W1.double(), W2.double()

    def near(got, ref):
        # two roundings to bf16 (result and intermediate): 2.4e-3 of the norm; a wrong row or plane is off by 1 or more
        assert ((got.double() - ref).norm() / ref.norm()).item() < 4e-3

    ends = [0, 1, 131071, 131072, 262143, 262144, 262145, M - 2, M - 1]  # (2^32 bytes are 262144 rows of P, 131072 of dP)
    p = [X[ends].double() @ w for w in w1]
    near(P[0][ends], p[0])
    near(P[1][ends], p[1])
    near(Y[ends], p[0] * torch.sigmoid(p[0]) * p[1] @ w2)
    r1, r2 = torch.zeros_like(w1), torch.zeros_like(w2)
    for at in range(0, M, 30000):
        rows = slice(at, min(M, at + 30000))
        g, u, d = P[0][rows].double(), P[1][rows].double(), dY[rows].double() @ w2.t()
        s = torch.sigmoid(g)
        dg, du = d * u * (s + g * s * (1 - s)), d * g * s
        if at in (0, 240000, 330000 // 30000 * 30000):
            near(dX[rows], dg @ w1[0].t() + du @ w1[1].t())
        x = X[rows].double()
        r1[0] += x.t() @ dg
        r1[1] += x.t() @ du
        r2 += (g * s * u).t() @ dY[rows].double()
    near(dW1, r1)
    near(dW2, r2)


def test_norm_rows_beyond_4_gb(lib):
    """140000 rows of 16384 bf16 (4.6 GB), a row stride of its own: the last rows against 64 bits."""
    M, H = 140001, 16384
    gen = torch.Generator(device="cuda").manual_seed(1)
    X = torch.empty((M, H + 8), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)[:, :H]
    Y, mean, rstd = torch.empty((M, H), dtype=torch.bfloat16, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    w, b = torch.randn(H, generator=gen, device="cuda"), torch.randn(H, generator=gen, device="cuda")
    plan = B.NormPlan(M, H, torch.bfloat16)
    plan.forward(X, w, b, Y, mean, rstd)
    dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    rows = [0, 131071, 131072, M - 1]
    x = X[rows].double()
    m = x.mean(1, keepdim=True)
    r = ((x - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    n = (x - m) * r
    assert ((Y[rows].double() - (n * w + b)).norm() / (n * w + b).norm()).item() < 3e-3
    plan.backward(Y, X, w, mean, rstd, Y2 := torch.empty_like(Y), dw, db)
    dy = Y[rows].double()
    g = dy * w
    ref = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    assert ((Y2[rows].double() - ref).norm() / ref.norm()).item() < 3e-3
    sums = torch.zeros(H, dtype=torch.float64, device="cuda")
    for at in range(0, M, 20000):
        sums += Y[at:at + 20000].double().sum(0)
    assert ((db.double() - sums).abs() <= 1e-6 * M + 1e-5 * sums.abs()).all()
