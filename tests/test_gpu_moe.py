"""The mixture-of-experts layer on the GPU against fp64: types, activations, one token to the most, empty and repeated slots, NaN, graphs."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as M
from paper_2607_07862_amd import binding as B
from tests._mx import NAMES, act_tol, held
from tests._train import U16, U32, assert_within, bf16, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def weights(gen, E, H, F, act, w):
    """The experts' weights as the plan takes them, and fp64 functions expert -> ([W1 ...], W2)."""
    nb = 2 if act == B.ACT_SWIGLU else 1
    W1, W2 = bf16(gen, (E, nb, H, F), H**-0.5).cuda(), bf16(gen, (E, F, H), F**-0.5).cuda()
    if w == "bf16":
        return W1, W2, lambda e: ([f64(W1[e, i]) for i in range(nb)], f64(W2[e]))
    a, b = B.MxMatrix(F, H, E * nb), B.MxMatrix(H, F, E)
    B.mx_quantize(W1.view(E * nb, H, F), a, down=True)
    B.mx_quantize(W2, b, down=True)
    return a, b, lambda e: ([held(a, e * nb + i).T for i in range(nb)], held(b, e).T)


def expected(X, ids, gates, of, E, name):
    """Y and its bounds.  Each expert's Z, after sums that are off by at most (H + 8) 2^-24 of their terms, is held as two bf16 numbers,
    the second a rounding (2^-8) of what the first left (at most 2^-8 of Z); its second product is off by (2 F + 40) 2^-24 of its terms, two
    for each of Z; the weighted sum adds a rounding a slot and the output's own."""
    T, H = X.shape
    Y, tol = np.zeros((T, H)), np.zeros((T, H))
    for e in range(E):
        token, slot = np.nonzero(ids == e)
        if not len(token):
            continue
        W1, W2 = of(e)
        x, g = X[token], gates[token, slot][:, None]
        p = [x @ w for w in W1]
        dp = [(x.shape[1] + 8) * U32 * (np.abs(x) @ np.abs(w)) for w in W1]
        z = M.act(name, p)
        dz = act_tol(name, p, dp)
        F = z.shape[1]
        y, mag = z @ W2, np.abs(z) @ np.abs(W2)
        off = (1 + U16) * (dz @ np.abs(W2)) + U16 * U16 * mag + (2 * F + 40) * (1 + U16) * U32 * mag
        np.add.at(Y, token, g * y)
        np.add.at(tol, token, np.abs(g) * (off + 16 * U32 * mag))
    return Y, tol + U16 * (np.abs(Y) + tol) + 1e-37


def case(T, H, F, E, k, act, w="bf16", router=BF, seed=0, plan=None, max_tokens=None):
    gen = torch.Generator().manual_seed(seed + 7 * T + H + E)
    X, Wr = bf16(gen, (T, H)).cuda(), (torch.randn((H, E), generator=gen) * H**-0.5).to(router).cuda()
    W1, W2, of = weights(gen, E, H, F, act, w)
    plan = plan or B.MoePlan(max_tokens or T, H, F, E, k, act, "mxfp4" if w == "mxfp4" else BF)
    return plan, X, Wr, W1, W2, of


def outputs(T, H, k):
    return (torch.full((T, H), float("nan"), dtype=BF, device="cuda"), torch.full((T, k), -7, dtype=torch.int32, device="cuda"),
            torch.full((T, k), float("nan"), device="cuda"))


def check(T, H, F, E, k, act, w="bf16", router=BF, **kw):
    plan, X, Wr, W1, W2, of = case(T, H, F, E, k, act, w, router, **kw)
    Y, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    want_ids, want = M.route(f64(X) @ f64(Wr), k)
    assert (ids.cpu().numpy() == want_ids).all(), "ids"
    assert_within(gates, want, 16 * U32 * np.ones_like(want), "gates")  # an exponential of 2 ulp, k additions, a division
    ref, tol = expected(f64(X), want_ids, want, of, E, NAMES[act])
    assert_within(Y, ref, tol, "Y")
    # the experts alone, with the router's choice
    again = torch.full_like(Y, float("nan"))
    plan.experts(X, ids, gates, W1, W2, again)
    assert torch.equal(again, Y)
    return plan


@pytest.mark.parametrize("w", ["bf16", "mxfp4"])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("T,H,F,E,k", [(1, 64, 64, 1, 1), (1, 128, 192, 8, 2), (2, 192, 64, 3, 3), (7, 320, 448, 16, 4), (16, 256, 128, 5, 2), (17, 128, 320, 6, 3),
                                       (33, 64, 256, 4, 2), (100, 192, 192, 3, 2)])
def test_sizes(lib, T, H, F, E, k, act, w):
    check(T, H, F, E, k, act, w)


@pytest.mark.parametrize("T,H,F,E,k,w,router", [(1, 2048, 1408, 64, 6, "bf16", F32), (1, 512, 2048, 8, 2, "mxfp4", BF), (3, 64, 64, 257, 16, "bf16", F32),
                                                (5, 128, 64, 512, 8, "mxfp4", BF), (128, 256, 128, 4, 4, "bf16", BF), (128, 128, 256, 4, 4, "mxfp4", F32),
                                                (300, 64, 128, 40, 9, "bf16", BF), (512, 128, 64, 8, 16 // 2, "mxfp4", BF), (1, 4096, 64, 300, 3, "bf16", F32)])
def test_larger(lib, T, H, F, E, k, w, router):
    check(T, H, F, E, k, B.ACT_SWIGLU, w, router)


@pytest.mark.parametrize("w", ["bf16", "mxfp4"])
@pytest.mark.parametrize("T,H,F,E,k,act", [(1, 2048, 1024, 3, 2, 2), (5, 1088, 2112, 6, 3, 1), (20, 2048, 1088, 3, 2, 0), (40, 1088, 1024, 3, 2, 2),
                                           (100, 1024, 2112, 2, 2, 1)])
def test_parts_of_k(lib, T, H, F, E, k, act, w):
    """Few items: K is cut in parts, with slots in lanes and slots counted in LDS."""
    check(T, H, F, E, k, act, w)


@pytest.mark.parametrize("T,H,E,k,router", [(300, 256, 9, 2, BF), (515, 256, 70, 4, F32), (1030, 256, 257, 2, BF), (2000, 64, 5, 4, F32), (8192, 64, 3, 1, BF)])
def test_many_tokens(lib, T, H, E, k, router):
    """One, two and four tokens to a work-group of the router; up to the most slots."""
    check(T, H, 64, E, k, B.ACT_IDENTITY, "bf16", router)


@pytest.mark.parametrize("w", ["bf16", "mxfp4"])
def test_largest_experts(lib, w):
    """H and F of 32768, the second expert: weights past 4 GB, with four elements that are not zero."""
    T, n = 3, 32768
    W1, W2 = torch.zeros((2, n, n), dtype=BF, device="cuda"), torch.zeros((2, n, n), dtype=BF, device="cuda")
    W1[1, n - 1, n - 1], W1[1, 0, n - 1] = 1, 2
    W2[1, n - 1, n - 1], W2[1, n - 1, 0] = 1, 3
    if w == "mxfp4":
        a, b = B.MxMatrix(n, n, 2), B.MxMatrix(n, n, 2)
        B.mx_quantize(W1, a, down=True)
        B.mx_quantize(W2, b, down=True)
        W1, W2 = a, b
    gen = torch.Generator().manual_seed(1)
    X = bf16(gen, (T, n)).cuda()
    ids, gates = torch.ones((T, 1), dtype=torch.int32, device="cuda"), torch.ones((T, 1), device="cuda")
    Y = torch.full((T, n), float("nan"), dtype=BF, device="cuda")
    B.MoePlan(T, n, n, 2, 1, B.ACT_IDENTITY, BF if w == "bf16" else "mxfp4").experts(X, ids, gates, W1, W2, Y)
    z = f64(X[:, n - 1]) + 2 * f64(X[:, 0])
    ref = np.zeros((T, n))
    ref[:, n - 1], ref[:, 0] = z, 3 * z
    assert_within(Y, ref, (U16 + 2 * U16 * U16) * np.abs(ref), "Y")  # the intermediate's two roundings (2^-16) and Y's


def test_fewer_tokens_than_planned(lib):
    plan = B.MoePlan(150, 128, 192, 10, 3, B.ACT_GELU_TANH)
    for T in (150, 1, 16, 17, 9, 64, 149, 2):
        check(T, 128, 192, 10, 3, B.ACT_GELU_TANH, plan=plan)
    plan.experts(*(torch.empty((0, n), dtype=t, device="cuda") for n, t in ((128, BF), (3, torch.int32), (3, F32))),
                 *weights(torch.Generator(), 10, 128, 192, 1, "bf16")[:2], torch.empty((0, 128), dtype=BF, device="cuda"))


@pytest.mark.parametrize("w", ["bf16", "mxfp4"])
@pytest.mark.parametrize("T", [1, 13, 90])
def test_empty_and_repeated_slots(lib, T, w):
    """Slots of -1 and of ids out of range, tokens with none, experts twice in a token, negative gates, NaN gates of empty slots."""
    E, k, H, F = 6, 4, 192, 128
    plan, X, _, W1, W2, of = case(T, H, F, E, k, B.ACT_SWIGLU, w)
    gen = torch.Generator().manual_seed(T)
    ids = torch.randint(-1, E, (T, k), generator=gen, dtype=torch.int32)
    gates = torch.randn((T, k), generator=gen)
    if T > 1:
        ids[1] = -1
        ids[2] = 3
        ids[3, :] = torch.tensor([E, -5, 1 << 30, 2], dtype=torch.int32)
        ids[T - 4:] = -1
    gates[(ids < 0) | (ids >= E)] = float("nan")
    Y = torch.full((T, H), float("nan"), dtype=BF, device="cuda")
    plan.experts(X, ids.cuda(), gates.cuda(), W1, W2, Y)
    ref, tol = expected(f64(X), ids.numpy(), gates.double().numpy(), of, E, "swiglu")
    assert_within(Y, ref, tol, "Y")
    if T > 1:
        assert (Y[1] == 0).all() and (Y[T - 4:] == 0).all()
    ids.fill_(-1)
    plan.experts(X, ids.cuda(), gates.cuda(), W1, W2, Y)
    assert (Y == 0).all()


def test_every_token_to_one_expert(lib):
    """All rows in one expert, more than one pass over its weights."""
    T, H, F, E, k = 200, 128, 192, 9, 2
    for w in ("bf16", "mxfp4"):
        plan, X, _, W1, W2, of = case(T, H, F, E, k, B.ACT_GELU_TANH, w)
        ids = torch.tensor([[7, 4]], dtype=torch.int32).repeat(T, 1)
        gates = torch.rand((T, k))
        Y = torch.empty((T, H), dtype=BF, device="cuda")
        plan.experts(X, ids.cuda(), gates.cuda(), W1, W2, Y)
        ref, tol = expected(f64(X), ids.numpy(), gates.double().numpy(), of, E, "gelu")
        assert_within(Y, ref, tol, w)


def test_ties_go_to_the_lowest_index(lib):
    T, H, E, k = 20, 256, 24, 6
    plan, X, Wr, W1, W2, _ = case(T, H, 64, E, k, B.ACT_SWIGLU, router=F32)
    Wr[:, 5] = Wr[:, 17] = Wr[:, 2]
    Wr[:, 11] = Wr[:, 3]
    X[4] = 0  # every logit equal
    Y, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    assert ids[4].tolist() == list(range(k)) and torch.allclose(gates[4], torch.full((k,), 1 / k, device="cuda"))
    for row in ids.tolist():
        at = {e: i for i, e in enumerate(row)}
        for low, high in ((2, 5), (5, 17), (3, 11)):
            assert high not in at or at[low] < at[high], row


def test_choice_between_logits_next_to_each_other(lib):
    """Columns of the router that differ in the last bit of one weight: fp32 sums would not tell them apart."""
    T, H, E, k = 64, 2048, 16, 8
    plan, X, Wr, W1, W2, _ = case(T, H, 64, E, k, B.ACT_SWIGLU, router=F32)
    Wr[:, 8:] = Wr[:, :8]
    for e in range(8, 16):
        Wr[100 + e, e] *= 1 + 2.0**-23
    Y, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    want, _ = M.route(f64(X) @ f64(Wr), k)
    assert (ids.cpu().numpy() == want).all()


def test_nan_and_infinity_stay_with_their_tokens(lib):
    T, H, F, E, k = 24, 128, 128, 8, 2
    plan, X, Wr, W1, W2, _ = case(T, H, F, E, k, B.ACT_SWIGLU)
    clean, ids0, gates0 = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, clean, ids0, gates0)
    X[3, 7], X[20, 0] = float("nan"), float("inf")
    Y, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    keep = [t for t in range(T) if t not in (3, 20)]
    assert torch.equal(Y[keep], clean[keep]) and torch.equal(ids[keep], ids0[keep])
    assert Y[3].isnan().all() and gates[3].isnan().all() and ids[3].tolist() == [0, 1]
    assert ((ids >= 0) & (ids < E)).all()
    # an expert's NaN weight reaches the tokens that chose it
    X[3], X[20] = 1, 1
    W2[5, 9, 100] = float("nan")
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    hit = (ids == 5).any(dim=1)
    assert hit.any() and torch.equal(Y.isnan().any(dim=1), hit) and Y[hit][:, 100].isnan().all()


@pytest.mark.parametrize("T", [1, 40])
def test_infinite_weight(lib, T):
    """An infinity in W2 makes its column infinite or NaN for the tokens that chose the expert, and nothing else."""
    H, F, E, k = 192, 128, 4, 2
    plan, X, Wr, W1, W2, _ = case(T, H, F, E, k, B.ACT_GELU_TANH)
    clean, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, clean, ids, gates)
    e = int(ids[0, 0])
    W2[e, 5, 70] = float("inf")
    Y = torch.full_like(clean, float("nan"))
    plan.experts(X, ids, gates, W1, W2, Y)
    hit = (ids == e).any(dim=1)
    assert not Y[hit][:, 70].isfinite().any()
    Y[hit, 70], clean[hit, 70] = 0, 0
    assert torch.equal(Y, clean)


def test_extreme_scales_of_weights(lib):
    """Scales 0 and 255 of a 4-bit expert: 2^-127, and NaN in the columns that have it."""
    T, H, F, E, k = 3, 128, 128, 2, 1
    plan, X, _, W1, W2, of = case(T, H, F, E, k, 0, "mxfp4")
    ids, gates = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.ones((T, k), device="cuda")
    W1.scales[0] = 127
    W2.scales[0, 0, :64] = 255
    W2.scales[0, 0, 64:] = 0
    Y = torch.zeros((T, H), dtype=BF, device="cuda")
    plan.experts(X, ids, gates, W1, W2, Y)
    assert Y[:, :64].isnan().all()
    (w1,), w2 = of(0)
    ref = M.act("identity", [f64(X) @ w1]) @ w2[:, 64:]
    assert_within(Y[:, 64:], ref, U16 * 8 * np.abs(ref).max() * np.ones_like(ref) + 2.0**-133, "Y")


def test_captured_and_beside_another_plan(lib):
    """A captured layer replays on new inputs, with another plan's calls on a second stream."""
    T, H, F, E, k = 20, 256, 320, 12, 3
    plan, X, Wr, W1, W2, _ = case(T, H, F, E, k, B.ACT_SWIGLU)
    other = B.MoePlan(T, H, F, E, k, B.ACT_SWIGLU)
    Y, ids, gates = outputs(T, H, k)
    plan.forward(X, Wr, W1, W2, Y, ids, gates)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.forward(X, Wr, W1, W2, Y, ids, gates)
    side = torch.cuda.Stream()
    want = outputs(T, H, k)
    for i in range(5):
        X.normal_()
        Y.zero_(), ids.zero_(), gates.zero_()
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        other.forward(X, Wr, W1, W2, *want, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(Y, want[0]) and torch.equal(ids, want[1]) and torch.equal(gates, want[2]), i


def test_rows_behind_the_last_are_left(lib):
    T, H, F, E, k = 5, 128, 64, 4, 2
    plan, X, Wr, W1, W2, _ = case(T, H, F, E, k, 1, max_tokens=9)
    Y, ids, gates = (torch.full((9, n), 3, dtype=t, device="cuda") for n, t in ((H, BF), (k, torch.int32), (k, F32)))
    plan.forward(X, Wr, W1, W2, Y[:T], ids[:T], gates[:T])
    assert (Y[T:] == 3).all() and (ids[T:] == 3).all() and (gates[T:] == 3).all()


def test_quantised_layer_end_to_end(lib):
    """As they are used together: a dense MLP's halves as 4-bit products with the activations quantised between, and the same
    weights as the only expert of a layer."""
    T, H, F = 24, 256, 512
    gen = torch.Generator().manual_seed(11)
    X = bf16(gen, (T, H)).cuda()
    W1, W2 = bf16(gen, (1, 2, H, F), H**-0.5).cuda(), bf16(gen, (1, F, H), F**-0.5).cuda()
    q1, q2, qx, qz = B.MxMatrix(F, H, 2), B.MxMatrix(H, F), B.MxMatrix(T, H), B.MxMatrix(T, F)
    B.mx_quantize(W1[0], q1, down=True)
    B.mx_quantize(W2, q2, down=True)
    Z, Y = torch.empty((T, F), dtype=BF, device="cuda"), torch.empty((T, H), dtype=BF, device="cuda")
    xv = torch.empty_like(X)
    B.mx_quantize(X, qx, values=xv)
    B.MxPlan(T, F, H, B.ACT_SWIGLU).product(qx, q1, Z)
    B.mx_quantize(Z, qz)
    B.MxPlan(T, H, F).product(qz, q2, Y)
    w1, w2 = [held(q1, i) for i in range(2)], held(q2)
    z = M.act("swiglu", [held(qx) @ w.T for w in w1])
    ref = held(qz) @ w2.T
    assert_within(Z, z, 2 * U16 * np.abs(z) + 1e-5, "Z")
    assert_within(Y, ref, U16 * np.abs(ref) + (F + 8) * U32 * (np.abs(held(qz)) @ np.abs(w2).T), "Y")
    plan = B.MoePlan(T, H, F, 1, 1, B.ACT_SWIGLU, "mxfp4")
    ids, gates = torch.zeros((T, 1), dtype=torch.int32, device="cuda"), torch.ones((T, 1), device="cuda")
    layer = torch.empty_like(Y)
    plan.experts(xv, ids, gates, q1, q2, layer)
    ref, tol = expected(f64(xv), ids.cpu().numpy(), f64(gates), lambda e: ([w.T for w in w1], w2.T), 1, "swiglu")
    assert_within(layer, ref, tol, "layer")
