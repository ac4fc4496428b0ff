"""A backward pass over no rows, whichever gradients are asked for."""
import pytest
import torch

from paper_2607_07862_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [B.ACT_IDENTITY, B.ACT_SWIGLU])
@pytest.mark.parametrize("asked", ["X", "1", "2", "X1", "X2", "12", "X12"])
def test_no_rows(lib, act, asked):
    H, F, nb = 64, 128, 2 if act == B.ACT_SWIGLU else 1
    new = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    plan = B.TrainPlan(4, H, F, act)
    W1, W2 = new(nb, H, F).zero_(), new(F, H).zero_()
    dX, dW1, dW2 = (t if c in asked else None for c, t in zip("X12", (new(0, H), new(nb, H, F), new(F, H))))
    plan.backward(new(0, H), new(0, H), W1, W2, new(nb, 0, F), dX, dW1, dW2)
    assert all(t is None or not t.any() for t in (dW1, dW2))


def test_no_gradient_is_still_refused(lib):
    plan = B.TrainPlan(4, 64, 128, B.ACT_IDENTITY)
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for M in (0, 2):
        with pytest.raises(B.Mlp2Error) as e:
            plan.backward(new(M, 64), new(M, 64), new(64, 128), new(128, 64), new(M, 128))
        assert e.value.code == B.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        plan.backward(new(0, 64), new(0, 64), new(64, 128), new(128, 64), new(0, 128), dX=new(0, 128))
