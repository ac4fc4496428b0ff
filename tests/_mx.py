"""Shared by the MXFP4 tests: matrices as the library stores them, and tolerances of products with activations.

Quantised values and their products are exact in fp32 (two significant bits and a power of two), so a product is off by its fp32 sum
alone, at most K 2^-24 sum |a w| (K + 8 is used), then by the activation's evaluation and the output's own rounding.
"""
from __future__ import annotations

import numpy as np
import torch

from oracle import mx_oracle as M
from tests._train import U16, U32, f64

NAMES = {0: "identity", 1: "gelu", 2: "swiglu"}


def stored(x: np.ndarray):
    """Codes and scales tensors [count, ...] (CPU) and the fp64 values [count, rows, K] of fp64 matrices [count, rows, K]."""
    codes, scales, values = [], [], []
    for m in x:
        c, s, v = M.quantise(m)
        c, s = M.pack(c, s)
        codes.append(c), scales.append(s), values.append(v[:, :m.shape[1]])
    return torch.from_numpy(np.ascontiguousarray(np.stack(codes))), torch.from_numpy(np.ascontiguousarray(np.stack(scales))), np.stack(values)


def held(m, i=0) -> np.ndarray:
    """fp64 values [rows, K] of matrix i of an MxMatrix."""
    return M.unpack(m.codes[i].cpu().numpy(), m.scales[i].cpu().numpy())[:, :m.K]


def act_tol(name, p, dp):
    """Bound of act's error where its pre-activations p are off by dp, before the output is rounded.

    The sigmoid takes 2^t of an argument rounded a few times: its relative error is within (4 |argument| + 8) 2^-24 (1 - s).  silu' and
    gelu' stay below 1.13."""
    if name == "identity":
        return dp[0]
    with np.errstate(over="ignore"):
        if name == "swiglu":
            s = 1 / (1 + np.exp(-p[0]))
            h = p[0] * s
            dh = 1.13 * dp[0] + np.abs(h) * U32 * ((1 - s) * (4 * np.abs(p[0]) + 8) + 4)
            return dh * (np.abs(p[1]) + dp[1]) + (np.abs(h)) * dp[1] + 2 * U32 * np.abs(h * p[1])
        y = 2 * np.sqrt(2 / np.pi) * (p[0] + 0.044715 * p[0] ** 3)
        s = 1 / (1 + np.exp(-y))
    v = np.abs(p[0] * s)
    return 1.13 * dp[0] + v * U32 * ((1 - s) * (8 * np.abs(y) + 8) + 4)


def product_and_tol(A, Ws, name, out32):
    """Y = act(A W^T) in fp64 and its bounds."""
    K = A.shape[1]
    p = [A @ w.T for w in Ws]
    dp = [(K + 8) * U32 * (np.abs(A) @ np.abs(w).T) for w in Ws]
    y = M.act(name, p)
    tol = act_tol(name, p, dp)
    return y, tol + (U32 if out32 else U16) * (np.abs(y) + tol) + 1e-37
