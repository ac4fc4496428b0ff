"""What the training operators launch, on the CPU: ``launch_log.cpp`` built for the host and asked.

A launch is a ``Launch``: kernel, the tile's rows and columns (0 where it has none), the epilogues' names, grid and block.
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

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


class Launch(NamedTuple):
    kernel: str
    tile: tuple
    stores: tuple
    grid: tuple
    block: int


@functools.lru_cache(maxsize=1)
def program() -> str | None:
    """The built program, or None where there is no compiler."""
    if not os.path.exists(HIPCC) or not shutil.which("c++filt"):
        return None
    folder = tempfile.mkdtemp(prefix="mlp2_launches_")
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    to = os.path.join(folder, "launch_log")
    cmd = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-no-hip-rt", "-std=c++17", "-O1",
           "-I" + os.path.join(ROOT, "paper_2607_07862_amd", "csrc"), "-I" + os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "launch_log.cpp"), "-o", to]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return to


def launches(*commands: str) -> list:
    """For each command (as ``launch_log.cpp`` documents them) its launches; every call has to succeed."""
    said = subprocess.run([program()], input="\n".join(commands) + "\n", stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
    assert len(said) == len(commands)
    out = []
    for command, line in zip(commands, said):
        words = line.split()
        assert words[0] == "0", (command, words[0])
        found = []
        for name, grid, block in zip(words[1::3], words[2::3], words[3::3]):
            full = demangled(name)
            t = [int(v) for v in m.group(1).split(",")] if (m := re.search(r"PTile<([\d, ]+)>", full)) else [0] * 4
            head = full.split("(")[0]
            found.append(Launch(re.search(r"k_\w+", full).group(), (t[0] * t[1], t[2] * t[3]), tuple(re.findall(r"Store\w+(?:<\w+>)?", head)),
                                tuple(int(v) for v in grid.split(",")), int(block)))
        out.append(found)
    return out


@functools.lru_cache(maxsize=None)
def demangled(name: str) -> str:
    return subprocess.run(["c++filt", name], stdout=subprocess.PIPE, text=True, check=True).stdout.strip()
