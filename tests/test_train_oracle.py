"""The training operators' fp64 oracle, pinned by differences and closed forms (CPU only)."""
import numpy as np
import pytest

from oracle import mlp2_oracle, train_oracle as T

ACTS = [T.ACT_IDENTITY, T.ACT_GELU_TANH, T.ACT_SWIGLU]


def problem(kind, M=5, H=6, F=7, seed=0):
    r = np.random.default_rng(seed)
    nb = 2 if kind == T.ACT_SWIGLU else 1
    return r.normal(size=(M, H)), r.normal(size=(nb, H, F)) / H**0.5, r.normal(size=(F, H)) / F**0.5, r.normal(size=(M, H))


def central(f, x, v, h=1e-5):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("kind", ACTS)
def test_mlp_gradients_are_the_differences_of_the_forward_pass(kind):
    X, W1, W2, dY = problem(kind)
    P, _ = T.mlp_forward(X, W1, W2, kind)
    dX, dW1, dW2, _, _ = T.mlp_backward(dY, X, W1, W2, P, kind)
    r = np.random.default_rng(1)
    for x, g, f in ((X, dX, lambda x: T.mlp_forward(x, W1, W2, kind)[1]), (W1, dW1, lambda w: T.mlp_forward(X, w, W2, kind)[1]),
                    (W2, dW2, lambda w: T.mlp_forward(X, W1, w, kind)[1])):
        for _ in range(4):
            v = r.normal(size=x.shape)
            assert np.isclose(central(lambda t: (f(t) * dY).sum(), x, v), (g * v).sum(), rtol=1e-7, atol=1e-8)


@pytest.mark.parametrize("kind", ACTS)
def test_mlp_forward_is_the_pinned_two_layer_product(kind):
    from paper_2607_07862_amd import inputs as I

    M, H, F = 4, 64, 64
    d = I.make_inputs(M, H, F, kind, 3)
    ref = mlp2_oracle.mlp2(I.bits(d["X"]), I.bits(d["W1"]), I.bits(d["W2"]), M, H, F, kind)
    W1 = d["W1"].double().numpy().reshape(-1, H, F)
    _, Y = T.mlp_forward(d["X"].double().numpy(), W1, d["W2"].double().numpy(), kind)
    assert np.allclose(Y, ref, rtol=1e-12, atol=1e-12)


def test_norm_gradients_are_the_differences_of_the_forward_pass():
    r = np.random.default_rng(2)
    X, w, b, dY, eps = r.normal(size=(4, 9)), r.normal(size=9), r.normal(size=9), r.normal(size=(4, 9)), 1e-3
    _, mean, rstd = T.norm_forward(X, w, b, eps)
    dX, dw, db = T.norm_backward(dY, X, w, mean, rstd)
    for x, g, f in ((X, dX, lambda x: T.norm_forward(x, w, b, eps)[0]), (w, dw, lambda t: T.norm_forward(X, t, b, eps)[0]),
                    (b, db, lambda t: T.norm_forward(X, w, t, eps)[0])):
        v = r.normal(size=x.shape)
        assert np.isclose(central(lambda t: (f(t) * dY).sum(), x, v), (g * v).sum(), rtol=1e-7, atol=1e-8)


def test_normalised_rows_have_no_mean_and_unit_variance():
    X = np.random.default_rng(3).normal(2.0, 3.0, size=(3, 50))
    Y, _, _ = T.norm_forward(X, np.ones(50), np.zeros(50), 0.0)
    assert np.allclose(Y.mean(1), 0) and np.allclose((Y**2).mean(1), 1)


@pytest.mark.parametrize("shape", [(6, 6), (4, 9), (9, 4), (1, 5), (5, 1), (1, 1)])
def test_ortho_acts_on_the_singular_values_alone(shape):
    G = np.random.default_rng(4).normal(size=shape)
    coeffs = [(3.4445, -4.7750, 2.0315)] * 5
    U, s, Vt = np.linalg.svd(G, full_matrices=False)
    t = s / np.linalg.norm(s)
    for a, b, c in coeffs:
        t = a * t + b * t**3 + c * t**5
    assert np.allclose(T.ortho(G, coeffs, 0.0), (U * t) @ Vt, atol=1e-10)


def test_cubic_coefficients_converge_to_the_orthogonal_factor():
    G = np.random.default_rng(5).normal(size=(5, 8))
    U, _, Vt = np.linalg.svd(G, full_matrices=False)
    assert np.allclose(T.ortho(G, [(1.5, -0.5, 0.0)] * 60, 0.0), U @ Vt, atol=1e-9)
