"""The MXFP4 and mixture-of-experts oracle against hand-derived values, exact arithmetic and plain loops (CPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import mx_oracle as M


def test_a_block_worked_by_hand():
    """Largest 7: 2^2 <= 7 < 2^3, scale 2^0; the rest by eye, ties to the even code."""
    x = np.zeros((1, 32))
    x[0, :14] = [7, -6.4, 5, -4.9, 3.5, 3.4, -2.5, 1.75, 1.25, 0.75, -0.25, 0.26, 1.6, -0.0]
    codes, scales, values = M.quantise(x)
    assert scales[0, 0] == 127
    assert values[0, :14].tolist() == [6, -6, 4, -4, 4, 3, -2, 2, 1, 1, 0, 0.5, 1.5, 0]
    assert codes[0, :14].tolist() == [7, 15, 6, 14, 6, 5, 12, 4, 2, 2, 8, 1, 3, 8]
    assert codes.shape == (1, 128) and (scales[0, 1:] == 0).all()


@pytest.mark.parametrize("top", [1.0, 1.999, 2.0**-126, 3e38, 2.0**-130, 6.0 * 2.0**-127])
def test_every_value_is_the_nearest_exactly(top):
    rng = np.random.default_rng(3)
    x = rng.uniform(-1, 1, (2, 32)) * top
    x[:, 0] = top
    codes, scales, values = M.quantise(x)
    for r in range(2):
        unit = Fraction(2) ** (int(scales[r, 0]) - 127)
        e = max(math.floor(math.log2(top)) - 2, -127)
        assert unit == Fraction(2) ** e
        for i in range(32):
            a = abs(Fraction(float(x[r, i])))
            best = min(abs(a - Fraction(float(g)) * unit) for g in M.GRID)
            assert abs(a - abs(Fraction(float(values[r, i])))) == best


def test_stored_arrays_give_the_values_back():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 200)) * np.exp(rng.standard_normal((5, 1)))
    codes, scales, values = M.quantise(x)
    packed, s = M.pack(codes, scales)
    assert packed.shape == (5, 128) and s.shape == (2, 5, 4)
    assert s[1, 3, 2] == scales[3, 6] and packed[4, 10] == codes[4, 20] + 16 * codes[4, 21]
    assert (M.unpack(packed, s) == values).all()


def test_blocks_with_nan_and_infinity():
    x = np.ones((1, 96))
    x[0, 5], x[0, 40] = np.nan, np.inf
    codes, scales, values = M.quantise(x)
    assert scales[0].tolist() == [255, 255, 125, 0]
    assert np.isnan(values[0, :64]).all() and (values[0, 64:96] == 1).all()


def test_route_and_experts_against_torch():
    g = torch.Generator().manual_seed(0)
    T, H, F, E, k = 7, 6, 10, 5, 3
    X, Wr = torch.randn((T, H), generator=g, dtype=torch.float64), torch.randn((H, E), generator=g, dtype=torch.float64)
    W1, W2 = torch.randn((E, 2, H, F), generator=g, dtype=torch.float64), torch.randn((E, F, H), generator=g, dtype=torch.float64)
    p = torch.softmax(X @ Wr, dim=1)
    top, ids = torch.topk(p, k, dim=1)
    top = top / top.sum(1, keepdim=True)
    got, gates = M.route((X @ Wr).numpy(), k)
    assert (got == ids.numpy()).all() and np.allclose(gates, top.numpy(), atol=1e-14)
    Y = torch.zeros((T, H), dtype=torch.float64)
    for e in range(E):
        Z = torch.nn.functional.silu(X @ W1[e, 0]) * (X @ W1[e, 1])
        Y += ((ids == e) * top).sum(1, keepdim=True) * (Z @ W2[e])
    assert np.allclose(M.experts(X.numpy(), got, gates, W1.numpy(), W2.numpy(), "swiglu"), Y.numpy(), atol=1e-12)
    p1 = torch.randn(9, generator=g, dtype=torch.float64)
    assert np.allclose(M.act("gelu", [p1.numpy()]), torch.nn.functional.gelu(p1, approximate="tanh").numpy(), atol=1e-14)


def test_ties_empty_slots_and_repeats():
    ids, gates = M.route(np.array([[1.0, 2.0, 2.0, 0.0]]), 2)
    assert ids.tolist() == [[1, 2]] and np.allclose(gates, 0.5)
    X, W1, W2 = np.ones((2, 1)), np.ones((2, 1, 1, 1)), np.array([[[3.0]], [[5.0]]])
    Y = M.experts(X, np.array([[0, -1], [1, 1]]), np.array([[1.0, 9.0], [0.25, 0.5]]), W1, W2, "identity")
    assert Y.tolist() == [[3.0], [3.75]]
