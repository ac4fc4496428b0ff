"""Plain fp64 NumPy definitions of the training operators (test infrastructure; shares no code with the HIP path).

* ``mlp_forward`` / ``mlp_backward``: ``P_i = X W1_i``, ``Z = act(P)``, ``Y = Z W2`` and its gradients;
* ``norm_forward`` / ``norm_backward``: layer norm over rows;
* ``ortho``: Newton-Schulz orthogonalisation of one matrix.

Arrays are float64; ``W1`` and ``P`` always carry a leading axis (one matrix, or gate and up).
"""
from __future__ import annotations

import numpy as np

ACT_IDENTITY, ACT_GELU_TANH, ACT_SWIGLU = 0, 1, 2


def _sigmoid(t):
    return 0.5 * (1.0 + np.tanh(0.5 * t))


def act(P, kind):
    """Z and the derivatives of Z with respect to each P_i."""
    if kind == ACT_IDENTITY:
        return P[0], [np.ones_like(P[0])]
    if kind == ACT_SWIGLU:
        s = _sigmoid(P[0])
        return P[0] * s * P[1], [P[1] * s * (1.0 + P[0] * (1.0 - s)), P[0] * s]
    k = np.sqrt(2.0 / np.pi)
    h = np.tanh(k * (P[0] + 0.044715 * P[0] ** 3))
    return 0.5 * P[0] * (1.0 + h), [0.5 * (1.0 + h) + 0.5 * P[0] * (1.0 - h * h) * k * (1.0 + 3 * 0.044715 * P[0] ** 2)]


def mlp_forward(X, W1, W2, kind):
    P = np.stack([X @ w for w in W1])
    return P, act(P, kind)[0] @ W2


def mlp_backward(dY, X, W1, W2, P, kind):
    """dX, dW1, dW2, and the intermediates (Z, dP) that tolerances are made of."""
    Z, slopes = act(P, kind)
    dZ = dY @ W2.T
    dP = np.stack([dZ * s for s in slopes])
    dX = sum(d @ w.T for d, w in zip(dP, W1))
    return dX, np.stack([X.T @ d for d in dP]), Z.T @ dY, Z, dP


def norm_forward(X, w, b, eps):
    mean = X.mean(axis=1)
    var = ((X - mean[:, None]) ** 2).mean(axis=1)
    rstd = 1.0 / np.sqrt(var + eps)
    return (X - mean[:, None]) * rstd[:, None] * w + b, mean, rstd


def norm_backward(dY, X, w, mean, rstd):
    xhat = (X - mean[:, None]) * rstd[:, None]
    g = dY * w
    dX = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dX, (dY * xhat).sum(axis=0), dY.sum(axis=0)


def ortho(G, coeffs, eps):
    """coeffs: one (a, b, c) per step."""
    X = G / (np.linalg.norm(G) + eps)
    for a, b, c in coeffs:
        S = X @ X.T if X.shape[0] <= X.shape[1] else X.T @ X
        B = b * S + c * S @ S
        X = a * X + (B @ X if X.shape[0] <= X.shape[1] else X @ B)
    return X
