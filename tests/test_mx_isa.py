"""ISA lint of the MXFP4 and mixture-of-experts kernels (CPU only), with the checks of ``test_train_isa``:

* no work-group barrier inside an exec-masked region;
* no scratch memory;
* the products' loops wait for their loads by their own counts, not by the compiler's;
* a direct-to-LDS load's scalar operands were not written by a vector instruction within five wait states, and M0 holds nothing else.
"""
import os
import re
import subprocess

import pytest

from test_isa_barriers import HIPCC, ROOT, mainloop_drains
from test_train_isa import code, kernels, masked_barriers, registers

SOURCES = ("mlp2_mx.hip", "mlp2_moe.hip")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    from paper_2607_07862_amd.build import CSRC, DEVICE_FLAGS

    out, runs = {}, []
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


def test_every_kernel_is_looked_at(asm):
    names = " ".join(kernels(asm))
    for k in ("k_mx_quantise_rows", "k_mx_quantise_down", "k_mx_product", "k_moe_route", "k_moe_bf16", "k_moe_mx"):
        assert k in names, k


def test_barriers_in_uniform_control_flow(asm):
    problems = {n: bad[:3] for n, b in kernels(asm).items() if (bad := masked_barriers(b))}
    assert not problems, problems


def test_no_scratch_memory(asm):
    for text in asm.values():
        sizes = dict(re.findall(r"\.name:\s+(_Z\w+)\n(?:.*\n)*?\s*\.private_segment_fixed_size: (\d+)", text))
        assert sizes and not {n: s for n, s in sizes.items() if int(s)}


def test_products_wait_for_their_loads_by_their_own_counts(asm):
    problems = {n: v[:3] for n, b in kernels(asm).items() if "k_mx_product" in n and (v := mainloop_drains(b))}
    assert not problems, problems


def load_hazards(lines):
    """Direct-to-LDS loads, of 16 or 4 bytes a lane, that read a scalar register too soon after a vector instruction wrote it."""
    bad, loads = [], 0
    for i, l in enumerate(lines):
        m = re.match(r"buffer_load_dword(?:x4)? v\d+, (s\[\d+:\d+\]), 0 offen(?: nt)? lds", l)
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
        if not lines[i - 1].startswith("s_nop"):
            bad.append(f"no wait state between M0 and {l}")
    return bad, loads


def test_scalar_operands_of_direct_to_lds_loads(asm):
    total, problems = 0, {}
    for n, b in kernels(asm).items():
        bad, loads = load_hazards(code(b))
        total += loads
        if bad:
            problems[n] = bad[:3]
        if loads:
            uses = [l for l in code(b) if re.search(r"\bm0\b", l) and not re.match(r"s_\w+ m0,(?!.*\bm0\b)", l)]
            assert not uses, (n, uses[:3])
    assert total > 100 and not problems, problems


def test_the_load_check_sees_a_planted_hazard():
    text = "v_readfirstlane_b32 s9, v3\ns_mov_b32 m0, s4\ns_nop {}\nbuffer_load_dword v1, s[8:11], 0 offen lds"
    assert load_hazards(text.format(0).splitlines()) == (["v_readfirstlane_b32 s9, v3 before buffer_load_dword v1, s[8:11], 0 offen lds"], 1)
    assert load_hazards(text.format(4).splitlines()) == ([], 1)
