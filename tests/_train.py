"""Shared by the training operators' GPU tests: inputs, and tolerances derived from the roundings the kernels make.

bf16 keeps 8 significant bits: rounding a value to it moves it by at most 2^-8
of itself.  An output therefore is off by 2^-8 |y| for its own rounding; where
one operand of its product was rounded to bf16 (Z, dP), by up to 2^-8 of every
term on top.  Those errors are independent: with K terms t_k the sum is within
2^-8 min(sqrt(K), 3.5) sqrt(sum t_k^2), the lesser of the worst case (by
Cauchy-Schwarz) and six standard deviations (a rounding's is at most
2^-8 / sqrt(3)).  fp32 sums of K products add at most K 2^-24 sum |t_k|.
"""
from __future__ import annotations

import numpy as np
import torch

U16, U32 = 2.0**-8, 2.0**-24
ACT_NAMES = {0: "identity", 1: "gelu", 2: "swiglu"}


def f64(t) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def product_tol(y, A, B, rounded_operand):
    """Element bounds of y = A @ B, rounded to bf16; A in fp32 or, if ``rounded_operand``, rounded to bf16 before."""
    K = A.shape[1]
    tol = U16 * np.abs(y) + (K + 8) * U32 * (np.abs(A) @ np.abs(B))
    if rounded_operand:
        tol = tol + 1.02 * U16 * min(K**0.5, 3.5) * np.sqrt((A * A) @ (B * B))
    return tol + 1e-37


def assert_within(got, ref, tol, what):
    g = f64(got)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    bad = ~(np.abs(g - ref) <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} elements out of bounds, first at {tuple(np.argwhere(bad)[0])}, worst {np.nanmax(np.abs(g - ref) / tol):.3g} times the bound"


def bf16(gen, shape, std=1.0):
    return (torch.randn(shape, generator=gen) * std).to(torch.bfloat16)
