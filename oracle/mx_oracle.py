"""Plain fp64 NumPy implementations of MXFP4 and of the mixture-of-experts layer (test infrastructure; shares no code with the HIP path).

MXFP4: 32 neighbours share a scale 2^e with e = floor(log2 max|x|) - 2 (at least -127); each value is the nearest of 0, 0.5, 1, 1.5, 2,
3, 4, 6 times the scale, ties to the even code, 6 for what lies above.  A block with a NaN or an infinity is NaN.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x: np.ndarray):
    """Codes (uint8, one an element), scale bytes (one a block of 32) and values of fp64 rows [rows, K]; K is padded with zeros to 128."""
    rows, K = x.shape
    kp = -(-K // 128) * 128
    full = np.zeros((rows, kp))
    full[:, :K] = x
    blocks = full.reshape(rows, kp // 32, 32)
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    scales = np.zeros(blocks.shape[:2], dtype=np.uint8)
    values = np.zeros(blocks.shape)
    for r, b in np.ndindex(*scales.shape):
        v = blocks[r, b]
        if not np.isfinite(v).all():
            scales[r, b], values[r, b] = 255, np.nan
            continue
        largest = np.abs(v).max()
        e = max(int(np.frexp(largest)[1]) - 3, -127) if largest else -127
        a = np.ldexp(np.abs(v), -e)
        far = np.abs(a[:, None] - GRID)
        near = far.argmin(axis=1)  # the lower of two at the same distance
        for i in np.nonzero(np.isclose(far.min(axis=1), np.partition(far, 1, axis=1)[:, 1], rtol=0, atol=0))[0]:
            near[i] += near[i] % 2  # a tie: the even code
        sign = np.signbit(v)
        codes[r, b] = near + 8 * sign
        scales[r, b] = e + 127
        values[r, b] = np.ldexp(np.where(sign, -GRID[near], GRID[near]), e)
    return codes.reshape(rows, kp), scales, values.reshape(rows, kp)


def unpack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 values [rows, Kp] of the stored arrays, codes [rows, Kp / 2] and scales [Kp / 128, rows, 4]."""
    rows = codes.shape[0]
    nibbles = np.stack([codes & 15, codes >> 4], axis=2).reshape(rows, -1)
    v = np.where(nibbles & 8, -GRID[nibbles & 7], GRID[nibbles & 7])
    s = scales.transpose(1, 0, 2).reshape(rows, -1).astype(np.int64)
    unit = np.where(s == 255, np.nan, np.ldexp(1.0, np.where(s == 255, 0, s - 127)))
    return v * np.repeat(unit, 32, axis=1)


def pack(codes: np.ndarray, scales: np.ndarray):
    """The stored arrays of one code an element [rows, Kp] and one scale a block [rows, Kp / 32]."""
    rows, kp = codes.shape
    return codes[:, 0::2] | codes[:, 1::2] << 4, scales.reshape(rows, kp // 128, 4).transpose(1, 0, 2)


def act(name: str, p):
    """act of a list of one or two pre-activations (fp64)."""
    with np.errstate(over="ignore"):
        if name == "swiglu":
            return p[0] / (1.0 + np.exp(-p[0])) * p[1]
        if name == "gelu":
            return 0.5 * p[0] * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (p[0] + 0.044715 * p[0] ** 3)))
    return p[0]


def route(logits: np.ndarray, k: int):
    """The k largest of each row (ties: the lowest index first) and the softmax over them."""
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(logits, ids, axis=1)
    e = np.exp(top - top[:, :1])
    return ids, e / e.sum(axis=1, keepdims=True)


def experts(X, ids, gates, W1, W2, name: str):
    """Y = sum over the slots of a token of gate * act(x W1[e]) W2[e]; slots outside [0, E) are empty.  W1 [E][nb] and W2 [E] hold
    matrices [H, F] and [F, H]."""
    Y = np.zeros((X.shape[0], W2[0].shape[1]))
    for t, j in np.ndindex(*ids.shape):
        e = ids[t, j]
        if 0 <= e < len(W2):
            Y[t] += gates[t, j] * (act(name, [X[t] @ w for w in W1[e]]) @ W2[e])
    return Y
