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

from test_isa_barriers import HIPCC, ROOT, loop_headers, mainloop_drains, parse_blocks, successors

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


PAIR = r"(s\[\d+:\d+\])"


def masked_barriers(body):
    """Barriers reached with a mask saved by s_and_saveexec / s_or_saveexec that has not been restored, and loops around a
    barrier that are continued through the exec mask.  As ``test_isa_barriers.violations``, but a register pair that saves a new
    mask stands for that mask alone (these kernels hold several products, whose code uses the same pairs again)."""
    blocks, heads = parse_blocks(body), loop_headers(body)
    index = {l: k for k, (l, _) in enumerate(blocks)}
    entry, work, bad = {0: ((), ())}, [0], set()
    while work:
        i = work.pop()
        state, alias = list(entry[i][0]), dict(entry[i][1])

        def close(reg):
            r = alias.get(reg, reg)
            if r not in state:
                return False
            del state[len(state) - 1 - state[::-1].index(r):]
            return True

        def save(reg):
            for a in [a for a, r in alias.items() if a == reg or r == reg]:
                del alias[a]
            state.append(reg)

        for ins in blocks[i][1]:
            if m := re.match(rf"s_(?:or|andn2)_saveexec_b64\s+{PAIR},\s*{PAIR}", ins):
                if close(m.group(2)) or ins.startswith("s_or"):
                    save(m.group(1))
            elif m := re.match(rf"s_and_saveexec_b64\s+{PAIR}", ins):
                save(m.group(1))
            elif m := re.match(rf"s_xor_b64\s+{PAIR},\s*(?:exec,\s*{PAIR}|{PAIR},\s*exec)", ins):
                src = m.group(2) or m.group(3)
                if alias.get(src, src) in state:
                    alias[m.group(1)] = alias.get(src, src)
            elif m := re.match(rf"s_or_b64\s+exec,\s*exec,\s*{PAIR}", ins):
                close(m.group(1))
            elif ins.startswith("s_barrier") and state:
                bad.add(f"{blocks[i][0]}: s_barrier with {state} saved")
            elif (m := re.match(r"s_cbranch_exec(?:nz|z)\s+(\.LBB\w+)", ins)) and m.group(1) in heads:
                h = index[m.group(1)]
                if any(x.startswith("s_barrier") for b in blocks[min(h, i):max(h, i) + 1] for x in b[1]):
                    bad.add(f"{blocks[i][0]}: exec-masked loop around a barrier")
        for j in successors(blocks, i):
            if j not in entry:
                entry[j] = (tuple(state), tuple(sorted(alias.items())))
                work.append(j)
    return sorted(bad)


def test_barriers_in_uniform_control_flow(asm):
    problems = {n: bad[:3] for n, b in kernels(asm).items() if (bad := masked_barriers(b))}
    assert not problems, problems


def test_the_barrier_check_sees_a_planted_mask():
    """A kernel of its own: a barrier between a saved mask and its restore, and one behind it."""
    text = "v_cmp_eq_u32 vcc, 0, v0\n\ts_and_saveexec_b64 s[2:3], vcc\n\ts_cbranch_execz .LBB0_1\n\t{0}\n.LBB0_1:\n\ts_or_b64 exec, exec, s[2:3]\n\t{1}\n\ts_endpgm\n"
    assert masked_barriers(text.format("s_barrier", "s_nop 0"))
    assert not masked_barriers(text.format("s_nop 0", "s_barrier"))


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
