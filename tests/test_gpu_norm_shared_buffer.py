"""Layer norm on matrices that lie beside each other in one wider buffer: accepted where no element is shared, and refused
where one is."""
import pytest
import torch

from paper_2607_07862_amd import binding as B

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def data(M, H, dtype, count):
    gen = torch.Generator().manual_seed(M + H)
    return [torch.randn((M, H), generator=gen).to(dtype).cuda() for _ in range(count)]


@pytest.mark.parametrize("M,H,gap", [(37, 96, 0), (5, 513, 3), (1, 40, 0), (300, 1000, 1)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_columns_of_one_buffer(lib, M, H, gap, dtype):
    X, dY = data(M, H, dtype, 2)
    plan = B.NormPlan(M, H, dtype)
    w, b = torch.rand(H, device="cuda"), torch.rand(H, device="cuda")
    Y, dX, mean, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    plan.forward(X, w, b, Y, mean, rstd)
    plan.backward(dY, X, w, mean, rstd, dX)
    wide = torch.full((M, 4 * (H + gap)), -7.0, dtype=dtype, device="cuda")
    x, y, dy, dx = (wide[:, i * (H + gap):i * (H + gap) + H] for i in range(4))
    x.copy_(X), dy.copy_(dY)
    plan.forward(x, w, b, y)
    plan.backward(dy, x, w, mean, rstd, dx)
    assert torch.equal(x, X) and torch.equal(dy, dY) and torch.equal(y, Y) and torch.equal(dx, dX)
    for i in range(4):
        assert (wide[:, i * (H + gap) + H:(i + 1) * (H + gap)] == -7.0).all(), "wrote between the matrices"


def test_types_of_their_own(lib):
    """fp32 rows with bf16 rows beside them: the same pitch in bytes."""
    M, H = 19, 200
    X, = data(M, H, F32, 1)
    plan = B.NormPlan(M, H, F32, BF)
    Y = torch.empty((M, H), dtype=BF, device="cuda")
    plan.forward(X, None, None, Y)
    wide = torch.zeros((M, 2 * H), device="cuda")
    x, y = wide[:, :H], wide.view(BF)[:, 2 * H:3 * H]
    x.copy_(X)
    plan.forward(x, None, None, y)
    assert torch.equal(x, X) and torch.equal(y, Y)


def test_rows_in_turn(lib):
    """X in the even rows of a buffer, Y in the odd ones."""
    M, H = 21, 130
    X, = data(M, H, BF, 1)
    plan = B.NormPlan(M, H, BF)
    Y = torch.empty_like(X)
    plan.forward(X, None, None, Y)
    both = torch.zeros((2 * M, H), dtype=BF, device="cuda")
    both[::2] = X
    plan.forward(both[::2], None, None, both[1::2])
    assert torch.equal(both[::2], X) and torch.equal(both[1::2], Y)


def refused(call, *args):
    with pytest.raises(B.Mlp2Error) as e:
        call(*args)
    assert e.value.code == B.ERR_INVALID_ARG


def test_shared_elements_are_refused(lib):
    M, H = 12, 50
    plan = B.NormPlan(M, H, BF)
    wide = torch.zeros((M + 2, 2 * H), dtype=BF, device="cuda")
    X = wide[:M, :H]
    st = torch.ones(M, device="cuda")
    for Y in (wide[:M, H - 1:2 * H - 1],                                        # one column
              wide[1:M + 1, :H],                                                # the rows after
              wide.view(-1)[2 * H - 1:].as_strided((M, H), (2 * H, 1)),         # a row's end over the next one's first element
              wide.view(-1)[H:].as_strided((M, H), (2 * H + 1, 1))):            # another pitch: rows drift into each other
        refused(plan.forward, X, None, None, Y)
        refused(plan.backward, wide.new_zeros((M, H)), X, None, st, st.clone(), Y)
    one = B.NormPlan(1, H, BF)
    flat = torch.zeros(2 * H, dtype=BF, device="cuda")
    refused(one.forward, flat[None, :H], None, None, flat[None, H - 1:2 * H - 1])
    one.forward(flat[None, :H], None, None, flat[None, H:])
    # the rows of X that Y's columns would meet are past the last
    plan.forward(wide[:M, :H], None, None, wide[:M, H:])
