"""Every tile of the training products against 64 bits: the 128 x 128 and 256 x 256 tiles with each epilogue, whole and in parts
of K, with ragged edges.  That the plans take these tiles for the shapes below is asserted on the CPU, from the launches.

The references are torch products of doubles on the GPU (two-dimensional ones); tolerances are those of the smaller shapes
(``_train``, ``test_gpu_ortho``)."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._launches import launches, program
from tests._train import U16, U32

GELU, SWIGLU = B.ACT_GELU_TANH, B.ACT_SWIGLU
# M, H, F, activation: tile rows (and columns) of P, Y, dZ and the shared launch, and the parts of K of P, Y and dZ
MLP = [
    (1024, 4096, 11008, SWIGLU, (256, 256, 256, 256), (1, 4, 1)),
    (500, 4096, 14336, SWIGLU, (256, 256, 256, 256), (1, 7, 2)),
    (500, 4096, 14336, GELU, (256, 256, 256, 256), (2, 7, 2)),
    (141, 5696, 17472, GELU, (256, 256, 256, 256), (3, 9, 3)),   # weight gradients of three stages, the last of 13 rows
    (4957, 256, 6336, SWIGLU, (256, 128, 256, 256), (1, 3, 1)),  # P and dZ of four stages
    (777, 2112, 5440, GELU, (128, 128, 128, 256), (1, 2, 1)),
    (2048, 1024, 2112, SWIGLU, (256, 64, 128, 128), (1, 1, 1)),
    (1500, 1024, 8192, SWIGLU, (256, 128, 256, 256), (1, 5, 1)),
]
# count, rows, cols, type: tile rows of A, B and X, and the parts of K of A, B and X
ORTHO = [
    (2, 2048, 2048, torch.float32, (128, 128, 128), (1, 1, 1)),
    (2, 2300, 1900, torch.bfloat16, (128, 128, 256), (1, 1, 1)),
    (1, 1900, 4100, torch.float32, (128, 64, 128), (2, 1, 1)),
    (4, 1664, 6656, torch.bfloat16, (256, 128, 256), (2, 1, 1)),
    (4, 6656, 1664, torch.float32, (256, 128, 256), (2, 1, 1)),
    (2, 3333, 5000, torch.float32, (256, 256, 256), (1, 1, 1)),
    (1, 20000, 1200, torch.float32, (128, 64, 256), (9, 1, 1)),
    (1, 4000, 14300, torch.bfloat16, (256, 256, 256), (1, 1, 1)),
    (1, 14300, 4000, torch.bfloat16, (256, 256, 256), (1, 1, 1)),
]
ids = lambda c: "x".join(str(v).replace("torch.", "") for v in c[:4])  # noqa: E731


def cdiv(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ the tiles, on the CPU


needs_compiler = pytest.mark.skipif(program() is None, reason="hipcc not available")


@needs_compiler
@pytest.mark.parametrize("M,H,F,act,tiles,parts", MLP, ids=map(ids, MLP))
def test_mlp_shapes_take_their_tiles(M, H, F, act, tiles, parts):
    forward, backward = launches(f"train {M} {H} {F} {act} {M} -", f"train {M} {H} {F} {act} {M} X12")
    found = forward + backward
    assert tuple(l.tile[0] for l in found) == tiles
    wide = [2 * F if act == SWIGLU else F, H, F]
    count = [cdiv(M, l.tile[0]) * cdiv(n, l.tile[1]) for l, n in zip(found, wide)]
    transposes = H // 64 * cdiv(M, 64)
    assert [l.grid[0] - (transposes if i == 2 else 0) for i, l in enumerate(found[:3])] == [n * p for n, p in zip(count, parts)]


@needs_compiler
def test_the_shape_of_three_stages_has_whole_weight_gradients():
    """Of the shared launch's items those of dX alone are in parts (few enough that the weight gradients' tiles could not be cut
    in two): the weight gradients run 141 rows, three stages, at once."""
    M, H, F, act = MLP[3][:4]
    shared, tile = launches(f"train {M} {H} {F} {act} {M} X12")[0][1], 256
    each, dx = cdiv(H, tile) * cdiv(F, tile), cdiv(M, tile) * cdiv(H, tile)
    rest = shared.grid[0] - 2 * each
    assert cdiv(M, 64) == 3 and rest % dx == 0 and 1 <= rest // dx <= 32 and rest < each


@needs_compiler
@pytest.mark.parametrize("count,rows,cols,dtype,tiles,parts", ORTHO, ids=map(ids, ORTHO))
def test_ortho_shapes_take_their_tiles(count, rows, cols, dtype, tiles, parts):
    found = launches(f"ortho {count} {rows} {cols} {B.DTYPE_F32 if dtype == torch.float32 else B.DTYPE_BF16} 5")[0][2:]
    assert len(found) == 15 and [l.stores[0] for l in found[-3:]] == ["StoreGram", "StorePoly", f"StoreLast<{str(rows > cols).lower()}>"]
    n, m = sorted(cdiv(v, 64) * 64 for v in (rows, cols))
    for i, l in enumerate(found):
        assert l.tile == (tiles[i % 3],) * 2 and l.grid[1] == count
        r = cdiv(n, l.tile[0])
        assert l.grid[0] == parts[i % 3] * (r * cdiv(m, l.tile[1]) if i % 3 == 2 else r * (r + 1) // 2)


# ------------------------------------------------------------------ their values, on the GPU


def near(got, ref, tol, what):
    assert got.shape == ref.shape
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at {tuple(bad.nonzero()[0].tolist())}, worst {(off / tol).max().item():.3g}"


def tol(y, A, W, rounded):
    """``_train.product_tol`` on the GPU: the bounds of y = A @ W for the roundings of its result, its sums and, if ``rounded``, of A."""
    K = A.shape[1]
    t = U16 * y.abs() + (K + 8) * U32 * (A.abs() @ W.abs()) + 1e-37
    return t + 1.02 * U16 * min(K**0.5, 3.5) * ((A * A) @ (W * W)).sqrt() if rounded else t


def product(got, A, W, rounded, what):
    y = A @ W
    near(got, y, tol(y, A, W, rounded), what)


def activation(p, act):
    """Z and its derivatives."""
    if act == SWIGLU:
        s = torch.sigmoid(p[0])
        return p[0] * s * p[1], [p[1] * s * (1 + p[0] * (1 - s)), p[0] * s]
    k = (2 / torch.pi) ** 0.5
    h = torch.tanh(k * (p[0] + 0.044715 * p[0] ** 3))
    return 0.5 * p[0] * (1 + h), [0.5 * (1 + h) + 0.5 * p[0] * (1 - h * h) * k * (1 + 3 * 0.044715 * p[0] ** 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,H,F,act,tiles,parts", MLP, ids=map(ids, MLP))
def test_mlp(lib, M, H, F, act, tiles, parts):
    gen = torch.Generator(device="cuda").manual_seed(M)
    normal = lambda std, *s: (torch.randn(s, generator=gen, device="cuda") * std).bfloat16()  # noqa: E731
    nb = 2 if act == SWIGLU else 1
    X, W1, W2, dY = normal(1.0, M, H), normal(H**-0.5, nb, H, F), normal(F**-0.5, F, H), normal(0.1, M, H)
    empty = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    P, Y, dX, dW1, dW2 = empty(nb, M, F), empty(M, H), empty(M, H), empty(nb, H, F), empty(F, H)
    plan = B.TrainPlan(M, H, F, act)
    plan.forward(X, W1, W2, P, Y)
    plan.backward(dY, X, W1, W2, P, dX, dW1, dW2)
    x, w2, dy, p = X.double(), W2.double(), dY.double(), P.double()
    w1 = [w.double() for w in W1]
    own = [x @ w for w in w1]
    for i in range(nb):
        near(P[i], own[i], tol(own[i], x, w1[i], False), f"P[{i}]")
    product(Y, activation(own, act)[0], w2, True, "Y")
    z, slopes = activation(p, act)
    dz = dy @ w2.t().contiguous()
    dp = [dz * s for s in slopes]
    product(dX, torch.cat(dp, 1), torch.cat([w.t() for w in w1]).contiguous(), True, "dX")
    xt = x.t().contiguous()
    for i in range(nb):
        y = xt @ dp[i]
        near(dW1[i], y, tol(y.t(), dp[i].t().contiguous(), x, True).t(), f"dW1[{i}]")
    product(dW2, z.t().contiguous(), dy, True, "dW2")


@pytest.mark.gpu
@pytest.mark.parametrize("count,rows,cols,dtype,tiles,parts", ORTHO, ids=map(ids, ORTHO))
def test_ortho(lib, count, rows, cols, dtype, tiles, parts):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    G = (1e-3 * torch.randn((count, rows, cols), generator=gen, device="cuda")).to(dtype)
    if count > 1:  # the stack's last one has a few strong directions
        left, right = torch.randn((rows, 8), generator=gen, device="cuda"), torch.randn((8, cols), generator=gen, device="cuda")
        G[-1] += (1e-2 * left @ right).to(dtype)
    O = torch.full(G.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    B.OrthoPlan(count, rows, cols, dtype).run(G, O)
    a, b, c = B.ORTHO_COEFFS
    for o, g in zip(O, G):
        x = g.double() if rows <= cols else g.double().t().contiguous()
        x = x / (torch.linalg.vector_norm(x) + 1e-7)
        for _ in range(5):
            s = x @ x.t().contiguous()
            x = a * x + (b * s + c * s @ s) @ x
        ref = x if rows <= cols else x.t()
        off, rms = (o.double() - ref).abs(), ref.square().mean().sqrt()
        assert off.norm() <= 3e-3 * ref.norm(), (off.norm() / ref.norm()).item()
        assert (off <= U16 * ref.abs() + 1.6e-2 * rms).all(), (off / rms).max().item()
