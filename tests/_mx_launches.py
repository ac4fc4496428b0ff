"""What the 4-bit products and the experts launch, on the CPU: ``mx_launch_log.cpp`` built for the host and asked.

The experts' items are counted on the device, from ids; ``work`` counts them here, by the formulas of ``Items`` in ``mlp2_moe.hip``.
"""
from __future__ import annotations

import atexit
import functools
import os
import re
import shutil
import subprocess
import tempfile
from typing import NamedTuple

import numpy as np

from tests._launches import HIPCC, ROOT, demangled


class Product(NamedTuple):
    choice: int  # the rows that choose() asked for: 64, 128, 256
    parts: int   # of K, as choose() asked for
    tile: tuple  # rows and columns of the kernel's tile
    groups: int  # work-groups
    block: int


class Experts(NamedTuple):
    kernel: str
    rows: int    # of an item, at most
    groups: int
    block: int
    blocks: int  # of columns
    steps: int   # of K
    most: int    # parts of K
    item: float
    join: float


class Work(NamedTuple):
    items: int
    parts: int
    per: int     # steps of a part; the last one may have fewer
    last: int    # steps of the last part


@functools.lru_cache(maxsize=1)
def program() -> str | None:
    """The built program, or None where there is no compiler."""
    if not os.path.exists(HIPCC) or not shutil.which("c++filt"):
        return None
    folder = tempfile.mkdtemp(prefix="mlp2_mx_launches_")
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    to = os.path.join(folder, "mx_launch_log")
    cmd = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-no-hip-rt", "-std=c++17", "-O1",
           "-I" + os.path.join(ROOT, "paper_2607_07862_amd", "csrc"), "-I" + os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "mx_launch_log.cpp"), "-o", to]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return to


def _said(commands):
    said = subprocess.run([program()], input="\n".join(commands) + "\n", stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
    assert len(said) == len(commands)
    for command, line in zip(commands, said):
        words = line.split()
        assert words[0] == "0", (command, words[0])
        yield words[1:]


def products(*shapes, cus: int = 256) -> list:
    """Of each (M, N, K, act, y dtype) its ``Product``."""
    out = []
    for words in _said([f"product {cus} {M} {N} {K} {act} {y} {M}" for M, N, K, act, y in shapes]):
        t = [int(v) for v in re.search(r"PTile<([\d, ]+)>", demangled(words[2])).group(1).split(",")]
        assert len(words) == 5
        out.append(Product(64 << int(words[0]), int(words[1]), (t[0] * t[1], t[2] * t[3]), int(words[3].split(",")[0]), int(words[4])))
    return out


def experts(*shapes, cus: int = 256) -> list:
    """Of each (max_tokens, H, F, E, k, act, w dtype, T) its two ``Experts``."""
    out = []
    for words in _said([f"experts {cus} " + " ".join(map(str, s)) for s in shapes]):
        found = []
        for name, grid, block, sizes in zip(*[iter(words)] * 4):
            full = demangled(name).split("(")[0]
            kernel, args = re.search(r"(k_moe_\w+)<(.*)>", full).groups()
            blocks, steps, most, item, join = sizes.split(",")
            found.append(Experts(kernel, 16 * int(args.split(",")[1]), int(grid.split(",")[0]), int(block), int(blocks), int(steps), int(most), float(item), float(join)))
        assert len(found) == 2
        out.append(found)
    return out


def work(e: Experts, ids: np.ndarray, E: int) -> Work:
    """The items of a product for these ids, and its parts of K."""
    f = np.float32
    count = np.bincount(ids[(ids >= 0) & (ids < E)].ravel(), minlength=E)
    units = int(sum(-(-c // e.rows) for c in count)) * e.blocks
    rounds = f(units) / f(e.groups)
    least, parts = f(1e30), 1
    for n in range(1, 17):
        steps = np.ceil(f(e.steps) * (f(1) / f(n)) - f(1e-3))
        cost = np.ceil(rounds * f(n) - f(1e-3)) * (steps + f(e.item)) + (f(e.join) * f(n) if n > 1 else f(0))
        if n <= e.most and cost < least:
            least, parts = cost, n
    per = -(-e.steps // parts)
    parts = -(-e.steps // per)
    return Work(units * parts, parts, per, e.steps - (parts - 1) * per)
