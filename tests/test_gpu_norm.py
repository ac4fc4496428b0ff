"""Layer norm on the GPU against the fp64 oracle: types, widths from one to the largest, odd widths and strides, offsets."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from paper_2607_07862_amd import binding as B
from tests._train import U16, U32, assert_within, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def case(M, H, x, y, pad=0, seed=0, offset=0.0):
    gen = torch.Generator().manual_seed(seed)
    wide = H + pad
    d = {"X": (torch.randn((M, wide), generator=gen) + offset).to(x), "dY": torch.randn((M, wide), generator=gen).to(y),
         "w": 1 + 0.2 * torch.randn(H, generator=gen), "b": torch.randn(H, generator=gen)}
    g = {k: v.cuda() for k, v in d.items()}
    g["X"], g["dY"] = g["X"][:, :H], g["dY"][:, :H]
    return g


def out(M, H, dtype, pad):
    return torch.full((M, H + pad), float("nan"), dtype=dtype, device="cuda")


def check(M, H, x, y, pad=0, out_pad=0, seed=0, offset=0.0, eps=1e-5, plan=None):
    """Tolerances: a mean or sum of H values in fp32 is within 8 2^-23 of the largest (pairwise sums of at most 16 in a row and
    10 levels); 1 / std scales that; bf16 results add 2^-8 of themselves, fp32 ones a few roundings."""
    g = case(M, H, x, y, pad, seed, offset)
    plan = plan or B.NormPlan(M, H, x, y)
    Y, mean, rstd = out(M, H, y, out_pad), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    plan.forward(g["X"], g["w"], g["b"], Y[:, :H], mean, rstd, eps=eps)
    X, dY, w, b = (f64(g[k]) for k in ("X", "dY", "w", "b"))
    rY, rm, rr = T.norm_forward(X, w, b, eps)
    big = np.abs(X).max(axis=1)
    fine = 8 * 2 * U32 * big  # of the mean, and of x - mean
    assert_within(mean, rm, fine, "mean")
    assert_within(rstd, rr, rr * (16 * U32 + 2 * fine * rr), "rstd")
    own = U16 if y == BF else 4 * U32
    xh = np.abs(X - rm[:, None]) * rr[:, None]
    near = (fine * rr)[:, None] * np.abs(w) * (1 + 2 * xh) + 16 * U32 * (xh * np.abs(w) + np.abs(b))
    assert_within(Y[:, :H], rY, own * np.abs(rY) + near, "Y")
    assert Y[:, H:].isnan().all(), "wrote past the rows"

    dX, dw, db = out(M, H, x, out_pad), torch.full((H,), float("nan"), device="cuda"), torch.full((H,), float("nan"), device="cuda")
    plan.backward(g["dY"], g["X"], g["w"], mean, rstd, dX[:, :H], dw, db)
    m, r = f64(mean), f64(rstd)
    rX, r_dw, r_db = T.norm_backward(dY, X, w, m, r)
    xh = (X - m[:, None]) * r[:, None]
    gw = dY * w
    own = U16 if x == BF else 4 * U32
    part = np.abs(gw) + np.abs(gw).mean(1, keepdims=True) + np.abs(xh) * np.abs(gw * xh).mean(1, keepdims=True)
    assert_within(dX[:, :H], rX, own * np.abs(rX) + r[:, None] * part * 32 * U32, "dX")
    assert dX[:, H:].isnan().all(), "wrote past the rows"
    assert_within(dw, r_dw, (M + 16) * U32 * np.abs(dY * xh).sum(0) + 1e-30, "dweight")
    assert_within(db, r_db, (M + 16) * U32 * np.abs(dY).sum(0) + 1e-30, "dbias")


@pytest.mark.parametrize("x,y", [(BF, BF), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("M,H", [(1, 1), (3, 1), (1, 4096), (5, 7), (2, 8), (70, 63), (9, 512), (9, 513), (300, 1024), (33, 1025), (17, 2048), (31, 2111),
                                 (1031, 640), (13, 4100), (6, 8192), (5, 8193), (4, 16384), (2, 16383)])
def test_both_passes_match_the_oracle(lib, M, H, x, y):
    check(M, H, x, y, seed=M + H)


@pytest.mark.parametrize("x,y", [(BF, BF), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("H,pad,out_pad", [(96, 32, 0), (513, 7, 3), (2111, 65, 1), (4096, 1, 5), (1000, 24, 8)])
def test_rows_of_any_stride(lib, H, pad, out_pad, x, y):
    check(37, H, x, y, pad, out_pad)


def test_more_rows_than_work_groups(lib):
    check(5000, 192, BF, BF)
    check(3001, 2100, F32, BF)


def test_rows_far_from_zero(lib):
    """A mean far above the spread: the variance is taken around the mean."""
    check(20, 1500, F32, F32, offset=1000.0)


def test_constant_rows_and_eps(lib):
    M, H = 6, 300
    plan = B.NormPlan(M, H, F32, F32)
    X = torch.arange(M, device="cuda", dtype=F32)[:, None].expand(M, H).contiguous()
    Y, mean, rstd = torch.empty_like(X), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    plan.forward(X, None, None, Y, mean, rstd, eps=1e-4)
    assert torch.allclose(mean, X[:, 0], rtol=1e-6) and torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-4)
    assert Y.abs().max() <= 100 * 8 * 2.0**-23 * M


def test_without_weight_bias_statistics_and_their_gradients(lib):
    M, H = 19, 700
    g = case(M, H, BF, BF)
    plan = B.NormPlan(M, H, BF)
    one, zero = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
    a, b = torch.empty_like(g["X"]), torch.empty_like(g["X"])
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    plan.forward(g["X"], one, zero, a, mean, rstd)
    plan.forward(g["X"], None, None, b)
    assert torch.equal(a, b)
    dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    plan.backward(g["dY"], g["X"], one, mean, rstd, a, dw, db)
    plan.backward(g["dY"], g["X"], None, mean, rstd, b)
    assert torch.equal(a, b)
    only = torch.empty(H, device="cuda")
    plan.backward(g["dY"], g["X"], one, mean, rstd, b, None, only)
    assert torch.equal(only, db)
    plan.backward(g["dY"], g["X"], one, mean, rstd, b, only, None)
    assert torch.equal(only, dw)


def test_no_rows_and_fewer_than_planned(lib):
    H = 260
    plan = B.NormPlan(64, H, BF)
    g = case(0, H, BF, BF)
    empty = torch.empty(0, device="cuda")
    plan.forward(g["X"], g["w"], g["b"], torch.empty_like(g["X"]), empty, empty)
    dw, db = torch.full((H,), float("nan"), device="cuda"), torch.full((H,), float("nan"), device="cuda")
    plan.backward(g["dY"], g["X"], g["w"], empty, empty, torch.empty_like(g["X"]), dw, db)
    assert not dw.any() and not db.any()
    for M in (64, 1, 40):
        check(M, H, BF, BF, plan=plan)


@pytest.mark.parametrize("H,rows", [(1000, (8, 9, 128, 129, 2, 264)), (64, (64, 65, 2048, 2049)), (1, (64, 2048, 2112)), (4093, (2, 3, 8, 10)), (16381, (1, 2))])
def test_weight_gradients_of_one_few_and_many_work_groups(lib, H, rows):
    """A work-group writes them alone, the last of few adds their parts, another kernel those of many: one plan, in turn."""
    plan = B.NormPlan(max(rows), H, BF)
    for M in rows + rows[:1]:
        check(M, H, BF, BF, seed=M, plan=plan)


@pytest.mark.parametrize("M,H", [(128, 1024), (2048, 64), (1024, 1024)])
def test_weight_gradients_have_the_same_bits_every_time(lib, M, H):
    g = case(M, H, BF, BF)
    plan = B.NormPlan(M, H, BF)
    Y, mean, rstd = torch.empty_like(g["X"]), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    plan.forward(g["X"], g["w"], g["b"], Y, mean, rstd)
    runs = []
    for _ in range(20):
        dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        plan.backward(g["dY"], g["X"], g["w"], mean, rstd, Y, dw, db)
        runs.append(torch.stack((dw, db)))
    assert all(torch.equal(runs[0], r) for r in runs[1:])


def test_a_bad_row_stays_alone(lib):
    M, H = 30, 900
    g = case(M, H, F32, F32)
    plan = B.NormPlan(M, H, F32)
    Y0, Y = torch.empty(M, H, device="cuda"), torch.empty(M, H, device="cuda")
    plan.forward(g["X"], g["w"], g["b"], Y0)
    g["X"][7, 3] = float("inf")
    g["X"][8, 5] = float("nan")
    plan.forward(g["X"], g["w"], g["b"], Y)
    keep = [i for i in range(M) if i not in (7, 8)]
    assert torch.equal(Y[keep], Y0[keep]) and Y[7].isnan().all() and Y[8].isnan().all()


def test_same_bits_each_run_and_on_another_stream(lib):
    M, H = 4000, 1024
    g = case(M, H, BF, BF)
    plan = B.NormPlan(M, H, BF)

    def both():
        Y, mean, rstd = torch.empty_like(g["X"]), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        plan.forward(g["X"], g["w"], g["b"], Y, mean, rstd)
        dX, dw, db = torch.empty_like(Y), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        plan.backward(g["dY"], g["X"], g["w"], mean, rstd, dX, dw, db)
        return Y, mean, rstd, dX, dw, db

    one = both()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        two = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, two))
