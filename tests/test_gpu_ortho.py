"""Newton-Schulz orthogonalisation on the GPU against the fp64 oracle: both orientations, odd sizes, stacks, hard spectra.

Tolerance: a bf16 result is off by 1.7e-3 of its norm through its own rounding.  The fp16 products add up to 2e-3 (a simulation
of their roundings in 64 bits over Gaussian, power-law, low-rank and rank-one matrices gave at most that, for the narrowest): 3e-3
of the norm allowed, and for single elements 2^-8 of themselves plus eight times 2e-3 of the root mean square."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from paper_2607_07862_amd import binding as B
from tests._train import U16, f64

pytestmark = pytest.mark.gpu
COEFFS = (3.4445, -4.7750, 2.0315)


def check(O, G, coeffs, eps=1e-7):
    for o, g in zip(f64(O), f64(G)):
        ref = T.ortho(g, coeffs, eps)
        off = np.abs(o - ref)
        rms = np.sqrt((ref**2).mean())
        assert np.linalg.norm(off) <= 3e-3 * np.linalg.norm(ref), np.linalg.norm(off) / np.linalg.norm(ref)
        assert (off <= U16 * np.abs(ref) + 1.6e-2 * rms).all(), (off / rms).max()


def run(G, plan=None, **kw):
    O = torch.full(G.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    (plan or B.OrthoPlan(*G.shape, G.dtype)).run(G, O, **kw)
    return O


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("count,rows,cols", [(1, 64, 64), (2, 128, 256), (1, 256, 128), (3, 65, 200), (1, 200, 65), (1, 63, 777), (2, 333, 31),
                                             (1, 512, 512), (1, 130, 1027), (1, 1027, 130), (4, 17, 16), (1, 700, 650)])
def test_matches_the_oracle(lib, count, rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows + cols)
    G = (1e-3 * torch.randn((count, rows, cols), generator=gen)).to(dtype).cuda()
    check(run(G), G, [COEFFS] * 5)


def spectrum(kind, n, m):
    r = np.random.default_rng(n + m)
    if kind == "rank one":
        return np.outer(r.normal(size=n), r.normal(size=m))
    if kind == "rank four and noise":
        return r.normal(size=(n, 4)) @ r.normal(size=(4, m)) + 1e-3 * r.normal(size=(n, m))
    s = 1.0 / np.arange(1, min(n, m) + 1) ** (1 if kind == "1 / k" else 2)
    U, V = np.linalg.qr(r.normal(size=(n, min(n, m))))[0], np.linalg.qr(r.normal(size=(m, min(n, m))))[0]
    return (U * s) @ V.T


@pytest.mark.parametrize("kind", ["rank one", "rank four and noise", "1 / k", "1 / k^2"])
@pytest.mark.parametrize("n,m", [(256, 256), (192, 600), (600, 192)])
def test_matrices_with_a_few_strong_directions(lib, kind, n, m):
    G = torch.from_numpy(spectrum(kind, n, m)).float().cuda()[None]
    check(run(G), G, [COEFFS] * 5)


def test_sizes_of_one(lib):
    for rows, cols in ((1, 1), (1, 300), (300, 1)):
        G = torch.randn((1, rows, cols), generator=torch.Generator().manual_seed(1)).cuda()
        check(run(G), G, [COEFFS] * 5)


@pytest.mark.parametrize("scale", [1e-12, 1e-3, 1e4, 1e12])
def test_any_scale_of_the_input(lib, scale):
    G = scale * torch.randn((1, 100, 140), generator=torch.Generator().manual_seed(2)).cuda()
    check(run(G, eps=1e-30), G, [COEFFS] * 5, eps=1e-30)


def test_steps_and_their_own_coefficients(lib):
    G = torch.randn((2, 90, 160), generator=torch.Generator().manual_seed(3)).cuda()
    own = [(3.9, -6.1, 3.0), (3.6, -5.0, 2.2), COEFFS, (1.875, -1.25, 0.375)]
    for coeffs in ([COEFFS], [COEFFS] * 2, own, [(1.5, -0.5, 0.0)] * 8):
        check(run(G, steps=len(coeffs), coeffs=coeffs), G, coeffs)


def test_zero_matrices_and_bad_values_stay_alone(lib):
    G = torch.randn((4, 70, 90), generator=torch.Generator().manual_seed(4)).cuda()
    plan = B.OrthoPlan(4, 70, 90, torch.float32)
    whole = run(G, plan)
    G[1] = 0.0
    G[2, 3, 4] = float("nan")
    got = run(G, plan)
    assert not got[1].any() and got[2].isnan().all()
    assert torch.equal(got[0], whole[0]) and torch.equal(got[3], whole[3])


def test_one_matrix_may_come_without_the_leading_axis_and_on_another_stream(lib):
    G = torch.randn((80, 48), generator=torch.Generator().manual_seed(5)).cuda()
    plan = B.OrthoPlan(1, 80, 48)
    a, b = torch.empty((80, 48), dtype=torch.bfloat16, device="cuda"), torch.empty((80, 48), dtype=torch.bfloat16, device="cuda")
    plan.run(G, a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    plan.run(G, b, stream=s)
    s.synchronize()
    assert torch.equal(a, b)
    check(a[None], G[None], [COEFFS] * 5)
