"""MLP training passes on the GPU against the fp64 oracle: every activation, row counts from one to several tiles, widths that
are multiples of 64 only, gradients left out, streams, repeated calls."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from paper_2607_07862_amd import binding as B
from tests._train import assert_within, bf16, f64, product_tol

pytestmark = pytest.mark.gpu


def case(M, H, F, act, seed=0):
    gen = torch.Generator().manual_seed(seed)
    nb = 2 if act == B.ACT_SWIGLU else 1
    d = {"X": bf16(gen, (M, H)), "W1": bf16(gen, (nb, H, F), H**-0.5), "W2": bf16(gen, (F, H), F**-0.5), "dY": bf16(gen, (M, H), 0.1)}
    return {k: v.cuda() for k, v in d.items()}


def forward(plan, g):
    P = torch.full((g["W1"].shape[0], g["X"].shape[0], plan.F), float("nan"), dtype=torch.bfloat16, device="cuda")
    Y = torch.full_like(g["X"], float("nan"))
    plan.forward(g["X"], g["W1"], g["W2"], P, Y)
    return P, Y


def backward(plan, g, P):
    out = [torch.full_like(g[k], float("nan")) for k in ("X", "W1", "W2")]
    plan.backward(g["dY"], g["X"], g["W1"], g["W2"], P, *out)
    return out


def check(plan, g, act):
    X, W1, W2, dY = (f64(g[k]) for k in ("X", "W1", "W2", "dY"))
    P, Y = forward(plan, g)
    ref, refY = T.mlp_forward(X, W1, W2, act)
    for i in range(W1.shape[0]):
        assert_within(P[i], ref[i], product_tol(ref[i], X, W1[i], False), f"P{i}")
    Z = T.act(ref, act)[0]
    assert_within(Y, refY, product_tol(refY, Z, W2, True), "Y")
    dX, dW1, dW2 = backward(plan, g, P)
    rX, r1, r2, Z, dP = T.mlp_backward(dY, X, W1, W2, f64(P), act)
    flat = np.concatenate(list(dP), axis=1), np.concatenate([w.T for w in W1], axis=0)
    assert_within(dX, rX, product_tol(rX, *flat, True), "dX")
    for i in range(W1.shape[0]):
        assert_within(dW1[i], r1[i], product_tol(r1[i].T, dP[i].T, X, True).T, f"dW1[{i}]")
    assert_within(dW2, r2, product_tol(r2, Z.T, dY, True), "dW2")


@pytest.mark.parametrize("act", [B.ACT_IDENTITY, B.ACT_GELU_TANH, B.ACT_SWIGLU])
@pytest.mark.parametrize("M,H,F", [(1, 64, 64), (2, 64, 192), (33, 128, 64), (64, 512, 1024), (65, 192, 320), (127, 448, 576),
                                   (130, 320, 1088), (257, 256, 512), (300, 832, 704), (700, 576, 832)])
def test_both_passes_match_the_oracle(lib, M, H, F, act):
    plan = B.TrainPlan(M, H, F, act)
    check(plan, case(M, H, F, act, M), act)


@pytest.mark.parametrize("M,H,F,act", [(2048, 1024, 2112, B.ACT_SWIGLU), (2500, 2048, 1024, B.ACT_GELU_TANH), (515, 4096, 4160, B.ACT_SWIGLU),
                                       (17, 4096, 6144, B.ACT_SWIGLU), (4097, 640, 512, B.ACT_IDENTITY)])
def test_large_products_match_the_oracle(lib, M, H, F, act):
    plan = B.TrainPlan(M, H, F, act)
    check(plan, case(M, H, F, act, M), act)


def test_fewer_rows_than_planned_and_repeated_calls(lib):
    plan = B.TrainPlan(300, 256, 320, B.ACT_SWIGLU)
    for M in (300, 5, 129, 300):
        g = case(M, 256, 320, B.ACT_SWIGLU, M)
        check(plan, g, B.ACT_SWIGLU)
        P, Y = forward(plan, g)
        again = forward(plan, g)
        assert torch.equal(P, again[0]) and torch.equal(Y, again[1])
        one, two = backward(plan, g, P), backward(plan, g, P)
        assert all(torch.equal(a, b) for a, b in zip(one, two))


def test_no_rows(lib):
    plan = B.TrainPlan(8, 128, 192, B.ACT_SWIGLU)
    g = case(0, 128, 192, B.ACT_SWIGLU)
    P, Y = forward(plan, g)
    dX, dW1, dW2 = backward(plan, g, P)
    assert Y.numel() == 0 and dX.numel() == 0
    assert not dW1.any() and not dW2.any()


@pytest.mark.parametrize("act", [B.ACT_IDENTITY, B.ACT_GELU_TANH, B.ACT_SWIGLU])
def test_gradients_that_are_not_asked_for(lib, act):
    M, H, F = 70, 192, 256
    plan = B.TrainPlan(M, H, F, act)
    g = case(M, H, F, act)
    P, _ = forward(plan, g)
    whole = backward(plan, g, P)
    for keep in ((0,), (1,), (2,), (0, 1), (1, 2)):
        out = [torch.zeros_like(t) if i in keep else None for i, t in enumerate(whole)]
        plan.backward(g["dY"], g["X"], g["W1"], g["W2"], P, *out)
        for i in keep:
            assert torch.equal(out[i], whole[i])


@pytest.mark.parametrize("act", [B.ACT_GELU_TANH, B.ACT_SWIGLU])
def test_gradients_are_the_differences_of_the_loss(lib, act):
    """<gradient, V> against the central difference of sum(Y dY) along V, both in 64 bits but for the GPU's gradient; each
    gradient's roundings move the inner product by at most 2^-7 of its terms' root sum of squares times six deviations."""
    M, H, F = 96, 128, 192
    plan = B.TrainPlan(M, H, F, act)
    g = case(M, H, F, act, 7)
    P, _ = forward(plan, g)
    grads = backward(plan, g, P)
    names = ("X", "W1", "W2")
    at = {k: f64(g[k]) for k in names}
    dY, r = f64(g["dY"]), np.random.default_rng(0)
    for name, grad in zip(names, grads):
        V, h = r.normal(size=at[name].shape), 1e-4
        loss = [(T.mlp_forward(**{**{"X": at["X"], "W1": at["W1"], "W2": at["W2"]}, name: at[name] + s * h * V}, kind=act)[1] * dY).sum() for s in (1, -1)]
        terms = f64(grad) * V
        # P was rounded to bf16 before the backward pass: another 2^-8 of each slope
        assert abs(terms.sum() - (loss[0] - loss[1]) / (2 * h)) <= 6 * 2.0**-7 * np.sqrt((terms**2).sum())


def test_saturated_activations(lib):
    """Pre-activations far in the tails: derivatives of exactly 0 and 1 side by side, no NaN."""
    M, H, F = 40, 64, 64
    for act in (B.ACT_GELU_TANH, B.ACT_SWIGLU):
        plan = B.TrainPlan(M, H, F, act)
        g = case(M, H, F, act)
        nb = g["W1"].shape[0]
        P = torch.tensor([0.0, -0.0, 20.0, -20.0, 120.0, -120.0, 3e4, -3e4]).repeat(nb * M * F // 8).view(nb, M, F).to(torch.bfloat16).cuda()
        if nb == 2:
            P[1] = 0.5
        dX, dW1, dW2 = backward(plan, g, P)
        X, W1, W2, dY = (f64(g[k]) for k in ("X", "W1", "W2", "dY"))
        rX, r1, r2, Z, dP = T.mlp_backward(dY, X, W1, W2, f64(P), act)
        flat = np.concatenate(list(dP), axis=1), np.concatenate([w.T for w in W1], axis=0)
        assert_within(dX, rX, product_tol(rX, *flat, True), "dX")
        for i in range(nb):
            assert_within(dW1[i], r1[i], product_tol(r1[i].T, dP[i].T, X, True).T, f"dW1[{i}]")
        assert_within(dW2, r2, product_tol(r2, Z.T, dY, True), "dW2")


def test_a_bad_row_spoils_only_what_it_feeds(lib):
    """A NaN row of X: its own rows of P, Y and dX and the weights' gradients are NaN, every other row is what it was."""
    M, H, F = 150, 128, 256
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    g = case(M, H, F, B.ACT_SWIGLU)
    P0, Y0 = forward(plan, g)
    dX0 = backward(plan, g, P0)[0]
    g["X"][149] = float("nan")
    P, Y = forward(plan, g)
    dX = backward(plan, g, P)[0]
    assert torch.equal(P[:, :149], P0[:, :149]) and torch.equal(Y[:149], Y0[:149]) and torch.equal(dX[:149], dX0[:149])
    assert Y[149].isnan().all() and dX[149].isnan().all()


def test_rows_past_the_end_are_never_read(lib):
    """M rows in front of a buffer of NaN: the ragged ends of every product, K of the weight gradients among them, read zeros."""
    M, H, F = 77, 192, 320
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    g = case(M, H, F, B.ACT_SWIGLU)
    P, Y = forward(plan, g)
    whole = backward(plan, g, P)
    for k in ("X", "dY"):
        wide = torch.full((M + 300, H), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:M] = g[k]
        g[k] = wide[:M]
    P2, Y2 = forward(plan, g)
    assert torch.equal(P, P2) and torch.equal(Y, Y2)
    assert all(torch.equal(a, b) for a, b in zip(whole, backward(plan, g, P2)))


def test_another_stream(lib):
    M, H, F = 200, 256, 384
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    g = case(M, H, F, B.ACT_SWIGLU)
    P, Y = forward(plan, g)
    whole = backward(plan, g, P)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        P2, Y2 = forward(plan, g)
        two = backward(plan, g, P2)
    s.synchronize()
    assert torch.equal(P, P2) and torch.equal(Y, Y2) and all(torch.equal(a, b) for a, b in zip(whole, two))


def test_graph_replays(lib):
    M, H, F = 48, 1024, 2048  # few rows: the calls that users capture, with K split over work-groups
    plan = B.TrainPlan(M, H, F, B.ACT_SWIGLU)
    g = case(M, H, F, B.ACT_SWIGLU)
    P = torch.empty((2, M, F), dtype=torch.bfloat16, device="cuda")
    Y = torch.empty_like(g["X"])
    out = [torch.empty_like(g[k]) for k in ("X", "W1", "W2")]
    graph = torch.cuda.CUDAGraph()
    plan.forward(g["X"], g["W1"], g["W2"], P, Y)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        plan.forward(g["X"], g["W1"], g["W2"], P, Y)
        plan.backward(g["dY"], g["X"], g["W1"], g["W2"], P, *out)
    for seed in range(4):
        g2 = case(M, H, F, B.ACT_SWIGLU, seed)
        P2, Y2 = forward(plan, g2)
        want = [P2, Y2] + backward(plan, g2, P2)
        torch.cuda.synchronize()
        for k in g:
            g[k].copy_(g2[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [P, Y] + out))
