"""The ping-pong loop of the training products (256 x 256 tiles): its ring protocol on the CPU, stage counts on the GPU.

The loop's slot program is read from the kernel source, as for the forward kernels' loops (``test_quad_ring``): for every stage
count no panel is read before every wave's pieces of it have arrived and a barrier has passed, and no ring slot is requested
again before every wave's reads of it are complete and a barrier has passed.
"""
import os
import re

import pytest

import test_quad_ring as Q

SRC = os.path.join(os.path.dirname(Q.SRC), "mlp2_product.hpp")


@pytest.fixture
def source(monkeypatch):
    monkeypatch.setattr(Q, "SRC", SRC)
    return tuple(t.replace("vm_wait(", "vm_traced(") for t in Q.loop_source("product_pingpong"))


def test_the_ring_protocol_for_every_stage_count(source):
    assert all(Q.check(source, nk, False, False) for nk in range(1, 14))


def test_no_looser_wait_keeps_the_ring_protocol(source):
    stage, rest = source
    waits = list(re.finditer(r"vm_traced\(int_constant<(.*?)>\(\)\)", stage))
    assert len(waits) == 4
    for m in waits:
        looser = stage[:m.start(1)] + re.sub(r"(?<=[?:] )\d+", lambda d: str(int(d.group()) + 2), m.group(1)) + stage[m.end(1):]
        with pytest.raises((AssertionError, KeyError)):
            for nk in range(1, 14):
                Q.check((looser, rest), nk, False, False)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [64, 128, 192, 256, 320, 1024])
def test_stage_counts_on_the_gpu(lib, K):
    """1000 rows through [K, 16384] and back: 256 x 256 tiles of one, two, three and more stages (and, for the weight gradients,
    a ragged last stage), against the same products in 64 bits."""
    import torch

    from paper_2607_07862_amd import binding as B
    from tests._train import assert_within, bf16, f64, product_tol

    M, F = 1000, 16384
    gen = torch.Generator().manual_seed(K)
    X, W1, W2, dY = bf16(gen, (M, K)).cuda(), bf16(gen, (1, K, F), K**-0.5).cuda(), bf16(gen, (F, K), F**-0.5).cuda(), bf16(gen, (M, K)).cuda()
    P, Y = torch.empty((1, M, F), dtype=torch.bfloat16, device="cuda"), torch.empty_like(X)
    plan = B.TrainPlan(M, K, F, B.ACT_IDENTITY)
    plan.forward(X, W1, W2, P, Y)
    ref = f64(X) @ f64(W1[0])
    assert_within(P[0], ref, product_tol(ref, f64(X), f64(W1[0]), False), "P")
    dX, dW1, dW2 = torch.empty_like(X), torch.empty_like(W1), torch.empty_like(W2)
    plan.backward(dY, X, W1, W2, P, dX, dW1, dW2)
    ref = f64(P[0]).T @ f64(dY)
    assert_within(dW2, ref, product_tol(ref, f64(P[0]).T, f64(dY), False), "dW2")
    dP = f64(dY) @ f64(W2).T
    ref = f64(X).T @ dP
    assert_within(dW1[0], ref, product_tol(ref.T, dP.T, f64(X), True).T, "dW1")
