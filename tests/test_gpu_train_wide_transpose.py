"""The transpose of an X with more 64 x 64 blocks than a launch has work-groups for it: 1048571 rows of 8256."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._launches import launches, program

M, H, F = (1 << 20) - 5, 8256, 64


@pytest.mark.skipif(program() is None, reason="hipcc not available")
def test_work_groups_take_two_blocks_each():
    with_x, without = launches(f"train {M} {H} {F} 0 {M} 1", f"train {M} {H} {F} 0 {M} 2")
    assert 2 * (with_x[0].grid[0] - without[0].grid[0]) == H // 64 * (-(-M // 64))


@pytest.mark.gpu
def test_weight_gradient_of_a_million_rows(lib):
    """Sums of -1, 0 and 1 over all rows: exact in fp32, so dW1 is the exact sum rounded to bf16."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    sign = lambda *s: torch.randint(-1, 2, s, generator=gen, dtype=torch.int8, device="cuda").bfloat16()  # noqa: E731
    X, dY = sign(M, H), torch.zeros((M, H), dtype=torch.bfloat16, device="cuda")
    dP = sign(M, F)
    dY[:, :F] = dP
    W1, W2, P = torch.zeros((H, F), dtype=torch.bfloat16, device="cuda"), torch.eye(F, H, device="cuda").bfloat16(), torch.zeros((M, F), dtype=torch.bfloat16, device="cuda")
    dW1 = torch.full((H, F), float("nan"), dtype=torch.bfloat16, device="cuda")
    plan = B.TrainPlan(M, H, F, B.ACT_IDENTITY)
    plan.backward(dY, X, W1, W2, P, dW1=dW1)
    sums = torch.zeros((H, F), dtype=torch.float64, device="cuda")
    for at in range(0, M, 40000):
        sums += X[at:at + 40000].double().t().contiguous() @ dP[at:at + 40000].double()
    assert torch.equal(dW1, sums.float().bfloat16())
