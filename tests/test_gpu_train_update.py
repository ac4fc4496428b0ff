"""The weights' update of the training example: orthogonalised momentum, scaled by each weight's fan-out over its fan-in."""
import pytest
import torch

from tests.test_gpu_train_block import example  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,F", [(256, 704), (320, 128)])
def test_the_update_scales_with_fan_out_over_fan_in(lib, example, H, F):  # noqa: F811
    """W1 is [2, H, F] and maps H to F, W2 is [F, H] and maps F to H (rows times W): where the output is the wider side the step
    grows by the root of the ratio, elsewhere it is the rate."""
    block = example.Block(32, H, F, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    for d in (block.d1, block.d2):
        d.copy_(torch.randn(d.shape, generator=gen, device="cuda") * 1e-2)
    block.dw.zero_(), block.db.zero_()
    before, rate = (block.W1.clone(), block.W2.clone()), 0.125
    block.update(rate)
    for W, was, o, fan_in, fan_out in ((block.W1, before[0], block.o1, H, F), (block.W2, before[1], block.o2, F, H)):
        step = rate * max(1.0, fan_out / fan_in) ** 0.5
        assert o.abs().max() > 0
        assert torch.allclose(W, was - step * o.float(), rtol=1e-5, atol=1e-6)
