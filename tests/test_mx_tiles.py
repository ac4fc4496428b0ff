"""The 4-bit product's 128 and 256 tiles against 64 bits, on random data: whole and in parts of K, several stages with a last one of fewer than
256 of K, ragged edges, more tiles than CUs (the largest tile's work-groups go on from tile to tile).  That these shapes take these tiles is
asserted on the CPU, from the launches."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._mx import NAMES, held as held_numpy
from tests._mx_gpu import assert_near, held, product_and_tol
from tests._mx_launches import products, program

BF, F32 = torch.bfloat16, torch.float32
ID, GELU, SWIGLU = B.ACT_IDENTITY, B.ACT_GELU_TANH, B.ACT_SWIGLU
# M, N, K, activation, type of Y: rows of the tile, parts of K
CASES = [
    (1000, 2111, 1100, ID, F32, 128, 1),
    (777, 3001, 1380, GELU, BF, 128, 1),
    (1000, 4100, 300, ID, BF, 128, 1),       # more tiles than CUs
    (600, 2111, 2400, SWIGLU, BF, 128, 1),
    (1000, 2111, 500, SWIGLU, F32, 128, 1),
    (500, 2111, 13000, GELU, F32, 128, 3),
    (600, 1100, 20000, SWIGLU, BF, 128, 2),
    (2111, 3001, 1100, SWIGLU, BF, 256, 1),
    (3000, 4100, 1100, GELU, BF, 256, 1),
    (1111, 4200, 2304, SWIGLU, F32, 256, 1),  # whole stages
    (3001, 4100, 1380, SWIGLU, BF, 256, 1),  # more tiles than CUs, from here on
    (2999, 8200, 1380, ID, F32, 256, 1),
    (4001, 6200, 1300, GELU, BF, 256, 1),
    (1000, 4100, 13000, GELU, BF, 256, 3),
    (500, 4100, 13000, SWIGLU, F32, 256, 3),
]
AHEAD = CASES[10:13]


def names(c):
    return "x".join(str(v) for v in c[:3]) + f"-{NAMES[c[3]]}-{str(c[4]).split('.')[1]}"


def cdiv(a, b):
    return -(-a // b)


@pytest.mark.skipif(program() is None, reason="hipcc not available")
def test_shapes_take_their_tiles():
    found = products(*[(M, N, K, act, B.DTYPE_F32 if y == F32 else B.DTYPE_BF16) for M, N, K, act, y, *_ in CASES])
    for (M, N, K, act, y, rows, parts), p in zip(CASES, found):
        tiles = cdiv(M, p.tile[0]) * cdiv(N, p.tile[1] // 2 if act == SWIGLU else p.tile[1])
        assert p.choice == rows and p.tile == (rows, rows) and p.parts == parts, (M, N, K, p)
        if (M, N, K, act, y, rows, parts) in AHEAD:
            assert tiles > 256 and tiles % 256 and p.groups == 256, (M, N, K, p, tiles)
        else:
            assert p.groups == tiles * parts, (M, N, K, p, tiles)


def matrix(gen, rows, K, count=1, std=1.0):
    x = torch.randn((count, rows, K), generator=gen, device="cuda") * torch.exp(0.5 * torch.randn((count, rows, 1), generator=gen, device="cuda")) * std
    mx = B.MxMatrix(rows, K, count)
    B.mx_quantize(x, mx)
    return mx


@pytest.mark.gpu
def test_values_of_the_reference(lib):
    """The GPU's reading of a matrix is the oracle's."""
    m = matrix(torch.Generator(device="cuda").manual_seed(1), 37, 300, 2)
    m.scales[0, 0, :6, 1] = torch.tensor([0, 1, 126, 200, 254, 255], dtype=torch.uint8, device="cuda")
    for i in range(2):
        assert torch.equal(held(m, i).cpu().nan_to_num(7.0), torch.from_numpy(held_numpy(m, i)).nan_to_num(7.0))


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,act,y,rows,parts", CASES, ids=map(names, CASES))
def test_product(lib, M, N, K, act, y, rows, parts):
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    nb = 2 if act == SWIGLU else 1
    A, W = matrix(gen, M, K), matrix(gen, N, K, nb, K**-0.5)
    whole = torch.full((M + 2, N), float("nan"), dtype=y, device="cuda")
    plan = B.MxPlan(M, N, K, act, y)
    plan.product(A, W, whole[:M])
    ref, tol = product_and_tol(held(A), [held(W, i) for i in range(nb)], NAMES[act], y == F32)
    assert_near(whole[:M], ref, tol, "Y")
    assert whole[M:].isnan().all()
    # new inputs in the same plan, and the same bits from the same ones
    again = torch.zeros((M, N), dtype=y, device="cuda")
    plan.product(A, W, again)
    assert torch.equal(again, whole[:M])
    B.mx_quantize(torch.randn((1, M, K), generator=gen, device="cuda"), A)
    plan.product(A, W, again)
    ref, tol = product_and_tol(held(A), [held(W, i) for i in range(nb)], NAMES[act], y == F32)
    assert_near(again, ref, tol, "Y of new inputs")
