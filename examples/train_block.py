"""Trains one pre-norm MLP block, ``y = x + mlp(norm(x))``, on a GPU: the training operators as they are used together.

A step runs layer norm and the gated MLP forward, the loss's gradient backward through both, and updates the MLP's weights
with their orthogonalised momentum (Muon); the norm's weight and bias take plain steps.  Plans are made once, outside the
loop, and every buffer is reused, so a step allocates nothing.  The target is what a block of other weights makes of
the same rows.

    python examples/train_block.py --tokens 2048 --width 512 --hidden 1408 --steps 60
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_07862_amd import binding as B  # noqa: E402


class Block:
    """Weights, gradients and plans of one block for up to ``rows`` rows of ``H`` elements (32-bit residual stream)."""

    def __init__(self, rows: int, H: int, F: int, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        bf16 = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.norm = B.NormPlan(rows, H, torch.float32, torch.bfloat16)
        self.mlp = B.TrainPlan(rows, H, F, B.ACT_SWIGLU)
        self.ortho1, self.ortho2 = B.OrthoPlan(2, H, F), B.OrthoPlan(1, F, H)
        self.weight, self.bias = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
        self.W1, self.W2 = normal(2, H, F) * H**-0.5, normal(F, H) * F**-0.5  # masters in 32 bits
        self.w1, self.w2 = self.W1.bfloat16(), self.W2.bfloat16()  # what the kernels read
        self.m1, self.m2 = torch.zeros_like(self.W1), torch.zeros_like(self.W2)
        self.d1, self.d2, self.o1, self.o2 = bf16(2, H, F), bf16(F, H), bf16(2, H, F), bf16(F, H)
        self.dw, self.db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        self.n, self.z, self.dn, self.P = bf16(rows, H), bf16(rows, H), bf16(rows, H), bf16(2, rows, F)
        self.mean, self.rstd, self.dx = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty((rows, H), device="cuda")

    def forward(self, x):
        self.norm.forward(x, self.weight, self.bias, self.n, self.mean, self.rstd)
        self.mlp.forward(self.n, self.w1, self.w2, self.P, self.z)
        return x + self.z

    def backward(self, x, dy):
        """Gradients of the weights, and of x (through the block and past it)."""
        self.mlp.backward(dy.bfloat16(), self.n, self.w1, self.w2, self.P, self.dn, self.d1, self.d2)
        self.norm.backward(self.dn, x, self.weight, self.mean, self.rstd, self.dx, self.dw, self.db)
        return dy + self.dx

    def update(self, rate: float, momentum: float = 0.9):
        for W, w, m, d, o, plan in ((self.W1, self.w1, self.m1, self.d1, self.o1, self.ortho1), (self.W2, self.w2, self.m2, self.d2, self.o2, self.ortho2)):
            m.mul_(momentum).add_(d)
            plan.run(m, o)
            fan_in, fan_out = W.shape[-2:]  # rows times W
            W.add_(o, alpha=-rate * max(1.0, fan_out / fan_in) ** 0.5)
            w.copy_(W)
        self.weight.add_(self.dw, alpha=-rate)
        self.bias.add_(self.db, alpha=-rate)


def train(tokens: int, width: int, hidden: int, steps: int, rate: float, say=print) -> list:
    """The loss (mean square over target's mean square) before each step and after the last."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((tokens, width), generator=gen, device="cuda")
    target = Block(tokens, width, hidden, seed=1).forward(x).clone()
    scale = (target - x).square().mean()
    block, losses = Block(tokens, width, hidden, seed=2), []
    for step in range(steps + 1):
        off = block.forward(x) - target
        losses.append((off.square().mean() / scale).item())
        if step % 10 == 0 or step == steps:
            say(f"step {step}: loss {losses[-1]:.4f}")
        if step < steps:
            block.backward(x, off * (2.0 / (tokens * width)))
            block.update(rate * (1.0 - step / steps))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1408)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rate", type=float, default=0.02)
    a = ap.parse_args()
    train(a.tokens, a.width, a.hidden, a.steps, a.rate)
