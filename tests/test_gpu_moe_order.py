"""The router's order where logits are NaN or infinite: NaN ahead of +infinity, ties to the lowest index, -infinity last."""
import pytest
import torch

from paper_2607_07862_amd import binding as B

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("router", [BF, F32])
@pytest.mark.parametrize("E,marks", [
    (8, {1: INF, 4: NAN}),
    (8, {0: INF, 2: NAN, 3: INF, 6: NAN, 7: -INF}),
    (70, {0: INF, 5: INF, 68: NAN, 69: INF, 33: -INF}),
    (300, {2: INF, 63: INF, 64: NAN, 127: NAN, 299: NAN, 0: -INF}),
    (4, {0: -INF, 1: -INF, 2: INF, 3: -INF}),
])
def test_nan_then_infinity(lib, E, marks, router):
    T, H, F = 5, 128, 64
    gen = torch.Generator().manual_seed(E)
    X = (torch.rand((T, H), generator=gen) + 0.5).to(BF).cuda()
    Wr = torch.randn((H, E), generator=gen)
    for e, v in marks.items():
        Wr[e % H, e] = v
    Wr = Wr.to(router).cuda()
    k = min(E, 16, len(marks) + 2)
    logits = (X.double() @ Wr.double()).cpu()
    want = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32)  # torch's order has NaN first
    assert all(want[:, i].tolist() == [e] * T for i, e in enumerate(sorted((e for e in marks if marks[e] != marks[e]))))
    W1, W2 = torch.randn((E, 2, H, F), dtype=BF, device="cuda"), torch.randn((E, F, H), dtype=BF, device="cuda")
    Y, ids, gates = torch.empty((T, H), dtype=BF, device="cuda"), torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    B.MoePlan(T, H, F, E, k).forward(X, Wr, W1, W2, Y, ids, gates)
    assert torch.equal(ids.cpu(), want)
    assert gates.isnan().all() and Y.isnan().all()  # softmax over NaN or +infinity
