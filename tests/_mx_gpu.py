"""References of the 4-bit products and the experts in 64 bits on the GPU, for sizes where NumPy takes too long: torch products of doubles, with
the bounds of ``_mx`` and of ``test_gpu_moe`` (the same formulas on tensors)."""
from __future__ import annotations

import torch

from tests._train import U16, U32

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def held(m, i=0) -> torch.Tensor:
    """fp64 values [rows, K] of matrix i of an MxMatrix."""
    codes, rows = m.codes[i], m.rows
    nibbles = torch.stack([codes & 15, codes >> 4], dim=2).view(rows, -1).int()
    table = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64, device=codes.device)
    s = m.scales[i].transpose(0, 1).reshape(rows, -1).double()
    unit = torch.where(s == 255, float("nan"), torch.exp2(s - 127))
    return (table[nibbles] * unit.repeat_interleave(32, dim=1))[:, :m.K].contiguous()


def act(name, p):
    if name == "swiglu":
        return p[0] * torch.sigmoid(p[0]) * p[1]
    if name == "gelu":
        return p[0] * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (p[0] + 0.044715 * p[0] ** 3))
    return p[0]


def act_tol(name, p, dp):
    """``_mx.act_tol``."""
    if name == "identity":
        return dp[0]
    if name == "swiglu":
        s = torch.sigmoid(p[0])
        h = p[0] * s
        dh = 1.13 * dp[0] + h.abs() * U32 * ((1 - s) * (4 * p[0].abs() + 8) + 4)
        return dh * (p[1].abs() + dp[1]) + h.abs() * dp[1] + 2 * U32 * (h * p[1]).abs()
    y = 2 * (2 / torch.pi) ** 0.5 * (p[0] + 0.044715 * p[0] ** 3)
    s = torch.sigmoid(y)
    return 1.13 * dp[0] + (p[0] * s).abs() * U32 * ((1 - s) * (8 * y.abs() + 8) + 4)


def product_and_tol(A, Ws, name, out32):
    """``_mx.product_and_tol``."""
    K = A.shape[1]
    ts = [w.t().contiguous() for w in Ws]
    p = [A @ t for t in ts]
    dp = [(K + 8) * U32 * (A.abs() @ t.abs()) for t in ts]
    y = act(name, p)
    tol = act_tol(name, p, dp)
    return y, tol + (U32 if out32 else U16) * (y.abs() + tol) + 1e-37


def experts_and_tol(X, ids, gates, of, E, name):
    """``test_gpu_moe.expected``: Y and its bounds; ids and gates on the GPU, of(e) an expert's ([W1 ...], W2) as [K, N]."""
    X, gates = X.double(), gates.double()
    Y, tol = torch.zeros_like(X), torch.zeros_like(X)
    for e in range(E):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if not len(token):
            continue
        W1, W2 = of(e)
        x, g = X[token], gates[token, slot][:, None]
        p = [x @ w for w in W1]
        dp = [(x.shape[1] + 8) * U32 * (x.abs() @ w.abs()) for w in W1]
        z = act(name, p)
        dz = act_tol(name, p, dp)
        y, mag, F = z @ W2, z.abs() @ W2.abs(), z.shape[1]
        off = (1 + U16) * (dz @ W2.abs()) + U16 * U16 * mag + (2 * F + 40) * (1 + U16) * U32 * mag
        Y.index_add_(0, token, g * y)
        tol.index_add_(0, token, g.abs() * (off + 16 * U32 * mag))
    return Y, tol + U16 * (Y.abs() + tol) + 1e-37


def assert_near(got, ref, tol, what):
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at {tuple(bad.nonzero()[0].tolist())}, worst {(off / tol).max().item():.3g}"
