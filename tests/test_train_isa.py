"""ISA lint of the training operators' kernels (CPU only), with the checks of ``test_isa_barriers``:

* no work-group barrier inside an exec-masked region;
* no scratch memory;
* the loops of matrix products wait for their loads by their own counts, not by the compiler's;
* a direct-to-LDS buffer load's scalar operands were not written by a vector instruction within five wait states (the loads
  are inline asm: the compiler keeps no wait states for them), and M0 holds nothing else.
"""
import os
import re
import subprocess

import pytest

from test_isa_barriers import HIPCC, ROOT, mainloop_drains, violations

SOURCES = ("mlp2_train.hip", "mlp2_norm.hip", "mlp2_ortho.hip")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    from paper_2607_07862_amd.build import CSRC, DEVICE_FLAGS

    out = {}
    runs = []
    for src in SOURCES:
        to = tmp_path_factory.mktemp("isa") / (src + ".s")
        cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--cuda-device-only", *DEVICE_FLAGS,
               "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, src), "-o", str(to)]
        runs.append((src, to, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, to, p in runs:
        said, _ = p.communicate()
        assert p.returncode == 0, said
        out[src] = to.read_text()
    return out


def kernels(asm):
    found = {}
    for text in asm.values():
        for m in re.finditer(r"^(_Z\w*\dk_\w+):", text, re.M):
            body = text[m.end():]
            found[m.group(1)] = body[:body.find(".Lfunc_end")]
    return found


def code(body):
    lines = (l.split(";")[0].strip() for l in body.splitlines())
    return [l for l in lines if l and not l.startswith((".", "#"))]


def test_every_kernel_is_looked_at(asm):
    names = " ".join(kernels(asm))
    for k in ("k_product", "k_products", "k_backward_first", "k_norm_forward", "k_norm_backward", "k_norm_reduce", "k_ortho_squares", "k_ortho_scale"):
        assert k in names, k


def test_barriers_in_uniform_control_flow(asm):
    problems = {n: bad[:3] for n, b in kernels(asm).items() if (bad := [v for v in violations(b) if "barrier" in v])}
    assert not problems, problems


def test_no_scratch_memory(asm):
    for text in asm.values():
        sizes = dict(re.findall(r"\.name:\s+(_Z\w+)\n(?:.*\n)*?\s*\.private_segment_fixed_size: (\d+)", text))
        assert sizes and not {n: s for n, s in sizes.items() if int(s)}


def test_mainloops_wait_for_their_loads_by_their_own_counts(asm):
    problems = {n: v[:3] for n, b in kernels(asm).items() if (v := mainloop_drains(b))}
    assert not problems, problems


def registers(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.match(r"s(\d+)$", operand)
    return {int(m.group(1))} if m else set()


def load_hazards(lines):
    bad, loads = [], 0
    for i, l in enumerate(lines):
        m = re.match(r"buffer_load_dwordx4 v\d+, (s\[\d+:\d+\]), 0 offen lds", l)
        if not m:
            continue
        loads += 1
        want, states = registers(m.group(1)), 0
        for prev in reversed(lines[max(0, i - 12):i]):
            if prev.startswith("s_nop"):
                states += int(prev.split()[1]) + 1
                continue
            if states >= 5:
                break
            if prev.startswith("v_") and any(registers(o.strip()) & want for o in prev.split(None, 1)[1].split(",")[:2]):
                bad.append(f"{prev} before {l}")
            states += 1
        if not re.match(r"s_nop", lines[i - 1]):
            bad.append(f"no wait state between M0 and {l}")
    return bad, loads


def test_direct_to_lds_loads_see_settled_scalars(asm):
    loads = 0
    for n, b in kernels(asm).items():
        bad, count = load_hazards(code(b))
        loads += count
        assert not bad, (n, bad[:3])
        for l in code(b):
            if "m0" in re.split(r"[\s,]+", l):
                assert re.match(r"s_\w+ m0,", l) and "m0" not in l.split(",", 1)[1], (n, l)
    assert loads > 100


def test_the_load_check_sees_a_planted_hazard():
    lines = ["v_readfirstlane_b32 s9, v1", "s_mov_b32 m0, s2", "s_nop 0", "buffer_load_dwordx4 v3, s[8:11], 0 offen lds"]
    assert load_hazards(lines)[0]
    assert not load_hazards(lines[:2] + ["s_nop 4"] + lines[3:])[0]
