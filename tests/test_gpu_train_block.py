"""The training operators together, as the example runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_block.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_a_block_lowers_its_loss(lib, example):
    """A block of random weights starts at a loss of about 2 (two independent outputs of the same size) and has to come well
    below what the best constant would give (1)."""
    losses = example.train(600, 256, 704, 40, 0.02, say=lambda s: None)
    assert 1.5 < losses[0] < 2.5 and losses[-1] < 0.5 and all(torch.isfinite(torch.tensor(losses)))


def test_the_step_is_the_gradient_of_the_loss(lib, example):
    """Central differences of the block's own loss along its input gradient, in 64 bits on the CPU, against the GPU's gradient."""
    import numpy as np

    from oracle import train_oracle as T
    from tests._train import f64

    rows, H, F = 90, 128, 192
    block = example.Block(rows, H, F, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, c = torch.randn((rows, H), generator=gen, device="cuda"), torch.randn((rows, H), generator=gen, device="cuda")
    block.forward(x)
    g = f64(block.backward(x, c))
    w1, w2, C = f64(block.w1), f64(block.w2), f64(c)

    def loss(t):
        n, _, _ = T.norm_forward(t, np.ones(H), np.zeros(H), 1e-5)
        return ((t + T.mlp_forward(n, w1, w2, T.ACT_SWIGLU)[1]) * C).sum()

    at, h = f64(x), 1e-4
    V = np.random.default_rng(0).normal(size=at.shape)
    terms = g * V
    # every element of g passed four bf16 roundings (dY, P, dP, dN): six deviations of their sum
    assert abs(terms.sum() - (loss(at + h * V) - loss(at - h * V)) / (2 * h)) <= 6 * 2.0**-7 * np.sqrt((terms**2).sum())
