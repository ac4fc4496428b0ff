"""One plan's captured and eager calls of different sizes in turn on one stream: the graphs and the eager calls share its workspace and counters."""
import pytest
import torch

from paper_2607_07862_amd import binding as B

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def captured(call):
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


@pytest.mark.parametrize("w", ["bf16", "mxfp4"])
def test_experts(lib, w):
    H, F, E, k, sizes = 1088, 2112, 9, 3, (150, 7, 40, 1)
    W1, W2 = torch.randn((E, 2, H, F), dtype=BF, device="cuda") * H**-0.5, torch.randn((E, F, H), dtype=BF, device="cuda") * F**-0.5
    Wr = torch.randn((H, E), device="cuda") * H**-0.5
    if w == "mxfp4":
        a, b = B.MxMatrix(F, H, 2 * E), B.MxMatrix(H, F, E)
        B.mx_quantize(W1.view(2 * E, H, F), a, down=True)
        B.mx_quantize(W2, b, down=True)
        W1, W2 = a, b
    new = lambda: B.MoePlan(max(sizes), H, F, E, k, B.ACT_SWIGLU, BF if w == "bf16" else w)  # noqa: E731
    plan, fresh = new(), [new() for _ in sizes]
    X = [torch.randn((T, H), dtype=BF, device="cuda") for T in sizes]
    out = [(torch.empty((T, H), dtype=BF, device="cuda"), torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")) for T in sizes]
    call = lambda p, i: p.forward(X[i], Wr, W1, W2, *out[i])  # noqa: E731
    graphs = [captured(lambda i=i: call(plan, i)) if i < 3 else None for i in range(len(sizes))]
    for turn in range(4):
        for x in X:
            x.normal_()
        want = []
        for i in range(len(sizes)):
            call(fresh[i], i)
            want.append([t.clone() for t in out[i]])
            [t.zero_() for t in out[i]]
        order = [(turn + j) % len(sizes) for j in range(len(sizes))]
        for i in order:  # no synchronisation between them
            graphs[i].replay() if graphs[i] else call(plan, i)
        torch.cuda.synchronize()
        for i in order:
            assert all(torch.equal(a, b) for a, b in zip(out[i], want[i])), (turn, sizes[i])


def test_product(lib):
    N, K, sizes = 520, 8300, (600, 16, 130, 1)
    W = B.MxMatrix(N, K, 2)
    B.mx_quantize(torch.randn((2, N, K), device="cuda") * K**-0.5, W)
    new = lambda: B.MxPlan(max(sizes), N, K, B.ACT_SWIGLU, F32)  # noqa: E731
    plan, fresh = new(), [new() for _ in sizes]
    A = [B.MxMatrix(M, K) for M in sizes]
    Y = [torch.empty((M, N), device="cuda") for M in sizes]
    graphs = []
    for i in range(len(sizes)):
        B.mx_quantize(torch.randn((sizes[i], K), device="cuda"), A[i])
        graphs.append(captured(lambda: plan.product(A[i], W, Y[i])) if i < 3 else None)
    for turn in range(4):
        want = []
        for i, M in enumerate(sizes):
            B.mx_quantize(torch.randn((M, K), device="cuda"), A[i])
            fresh[i].product(A[i], W, Y[i])
            want.append(Y[i].clone())
            Y[i].zero_()
        order = [(turn + j) % len(sizes) for j in range(len(sizes))]
        for i in order:
            graphs[i].replay() if graphs[i] else plan.product(A[i], W, Y[i])
        torch.cuda.synchronize()
        assert all(torch.equal(Y[i], want[i]) for i in order), turn
