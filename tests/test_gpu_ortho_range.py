"""Newton-Schulz orthogonalisation of inputs at both ends of fp32's range, where their squares are not in it.  Tolerances as
for inputs of ordinary size (``test_gpu_ortho``): the iteration does not know the input's scale."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests.test_gpu_ortho import COEFFS, check, run

pytestmark = pytest.mark.gpu


def normal(shape, scale, seed=0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale).clamp(-3.3e38, 3.3e38).float()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1e-40, 1e-30, 1e-24, 1e-20, 1e17, 1e20, 1e30, 1e36, 2e38])
@pytest.mark.parametrize("rows,cols", [(100, 140), (140, 100)])
def test_any_scale_without_eps(lib, rows, cols, scale, dtype):
    """(2e38: the norm itself, 2e40, is past fp32.  In bf16 1e-40 would be of one bit: taken in fp32 alone.)"""
    if dtype == torch.bfloat16 and scale < 1e-36:
        dtype = torch.float32
    G = normal((1, rows, cols), scale).to(dtype).cuda()
    check(run(G, eps=0.0), G, [COEFFS] * 5, eps=0.0)


def test_matrices_of_a_stack_have_scales_of_their_own(lib):
    G = torch.stack([normal((90, 130), s, i) for i, s in enumerate((1e-32, 1.0, 1e32, 1e-3))]).cuda()
    check(run(G, eps=1e-40), G, [COEFFS] * 5, eps=float(torch.tensor(1e-40)))


@pytest.mark.parametrize("eps", [1e-7, 1e-30])
def test_norms_around_eps(lib, eps):
    """|G| from a hundredth of eps to a hundred times it: the result shrinks with G / (|G| + eps)."""
    plan = B.OrthoPlan(1, 100, 140)
    for ratio in (0.01, 0.1, 1.0, 100.0):
        G = normal((1, 100, 140), ratio * eps / 118).cuda()
        check(run(G, plan, eps=eps), G, [COEFFS] * 5, eps=float(torch.tensor(eps)))


def test_zeros_and_infinities_are_what_they_were(lib):
    G = normal((4, 70, 90), 1e30).cuda()
    G[1] = 0.0
    G[2, 3, 4] = float("inf")
    got = run(G, eps=1e-7)
    assert not got[1].any() and got[2].isnan().all()
    check(got[[0, 3]], G[[0, 3]], [COEFFS] * 5)
