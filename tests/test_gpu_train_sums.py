"""What other tests compute on the way and do not look at: weight gradients beside a bad row, the norm's statistics and weight
gradient over more than 4 GB, graph replays of the norm and the orthogonalisation."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._train import U32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("act", [B.ACT_IDENTITY, B.ACT_GELU_TANH, B.ACT_SWIGLU])
def test_a_bad_row_reaches_every_weight_gradient(lib, act):
    M, H, F, nb = 150, 128, 256, 2 if act == B.ACT_SWIGLU else 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(BF)  # noqa: E731
    X, W1, W2, dY = normal(M, H), normal(nb, H, F), normal(F, H), normal(M, H)
    X[149] = float("nan")
    P, Y, dX, dW1, dW2 = normal(nb, M, F), torch.empty_like(X), torch.empty_like(X), torch.zeros_like(W1), torch.zeros_like(W2)
    plan = B.TrainPlan(M, H, F, act)
    plan.forward(X, W1, W2, P, Y)
    plan.backward(dY, X, W1, W2, P, dX, dW1, dW2)
    assert dW1.isnan().all() and dW2.isnan().all()


def test_norm_sums_over_more_than_4_gb(lib):
    """140001 rows of 16384 at a stride of their own: every mean, rstd and element of dweight and dbias against 64 bits."""
    M, H = 140001, 16384
    gen = torch.Generator(device="cuda").manual_seed(2)
    X = torch.empty((M, H + 8), dtype=BF, device="cuda").normal_(generator=gen)[:, :H]
    dY = torch.empty((M, H), dtype=BF, device="cuda").normal_(generator=gen)
    mean, rstd, dw, db = torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    w, out = torch.ones(H, device="cuda"), torch.empty((M, H), dtype=BF, device="cuda")
    plan = B.NormPlan(M, H, BF)
    plan.forward(X, w, None, out, mean, rstd)
    plan.backward(dY, X, w, mean, rstd, out, dw, db)
    sums = torch.zeros((4, H), dtype=torch.float64, device="cuda")
    for at in range(0, M, 10000):
        rows = slice(at, at + 10000)
        x, dy = X[rows].double(), dY[rows].double()
        m = x.mean(1)
        r = ((x - m[:, None]).square().mean(1) + 1e-5).rsqrt()
        fine = 8 * 2 * U32 * x.abs().amax(1)  # of a mean over H values in fp32
        assert ((mean[rows].double() - m).abs() <= fine).all()
        assert ((rstd[rows].double() - r).abs() <= r * (16 * U32 + 2 * fine * r)).all()
        t = dy * (x - mean[rows].double()[:, None]) * rstd[rows].double()[:, None]
        sums += torch.stack((t.sum(0), t.abs().sum(0), dy.sum(0), dy.abs().sum(0)))
    assert ((dw.double() - sums[0]).abs() <= (M + 16) * U32 * sums[1]).all()
    assert ((db.double() - sums[2]).abs() <= (M + 16) * U32 * sums[3]).all()
    # no sum of 140001 values in fp32 is off by more than the root of its count in roundings, six deviations
    assert ((dw.double() - sums[0]).abs() <= 6 * M**0.5 * U32 * sums[1]).all()


@pytest.mark.parametrize("M,H", [(16, 1000), (300, 1024), (1, 4096)])
def test_norm_graph_replays(lib, M, H):
    """One work-group, a join by the last of few, and another kernel's sum: each replay against a call outside the graph."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    X, dY, w, b = torch.empty((M, H), dtype=BF, device="cuda"), torch.empty((M, H), dtype=BF, device="cuda"), torch.rand(H, device="cuda"), torch.rand(H, device="cuda")
    plan = B.NormPlan(M, H, BF)

    def both():
        Y, dX, mean, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        plan.forward(X, w, b, Y, mean, rstd)
        plan.backward(dY, X, w, mean, rstd, dX, dw, db)
        return Y, mean, rstd, dX, dw, db

    X.normal_(generator=gen), dY.normal_(generator=gen)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for _ in range(4):
        X.normal_(generator=gen), dY.normal_(generator=gen)
        want = both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, kept))


@pytest.mark.parametrize("count,rows,cols", [(2, 100, 700), (1, 600, 300)])
def test_ortho_graph_replays(lib, count, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(4)
    G, O = torch.empty((count, rows, cols), device="cuda"), torch.empty((count, rows, cols), dtype=BF, device="cuda")
    plan = B.OrthoPlan(count, rows, cols)
    plan.run(G.normal_(generator=gen), O)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run(G, O)
    for _ in range(4):
        G.normal_(generator=gen)
        plan.run(G, want := torch.empty_like(O))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, O)
